// Which places of a tensor the kernels around the convolutions touch: index arithmetic without anything of the GPU's, so that it can be
// checked on the CPU at sizes that no test runs (tests/test_layers_index.py).
#pragma once

#include <cstdint>

namespace fftconv {
namespace lay {

// The weight's gradient reads the 64 samples from n0 on of a sequence of N in whole pieces of 16 bytes, or, where that would touch what the
// tensor does not have, piece by piece with its end looked at. dy (b, n, o) is read in pieces of 8 channels: the last piece of a sample's O
// channels reaches past them, into the samples after it as long as there are enough of those. (With less than 8 channels it may take several.)
__host__ __device__ inline bool whole_half_run(int64_t n0, int64_t N, int64_t O, bool tokens)
{
    const int64_t after = N - n0 - 64;                       // samples behind them
    return after >= 0 && (!tokens || after * O >= (O + 7) / 8 * 8 - O);
}

// A launch holds less than 2^32 threads (a longer one is cut short without an error): more workgroups go out in pieces, f(the first one's number,
// how many), until one of them returns a code other than 0.
template <typename F> inline int in_pieces(int64_t groups, int threads, F f)
{
    const int64_t most = (((int64_t)1 << 32) - 1) / threads;
    for (int64_t first = 0; first < groups; first += most)
        if (const int rc = f(first, (unsigned)(groups - first < most ? groups - first : most))) return rc;
    return 0;
}

}  // namespace lay
}  // namespace fftconv
