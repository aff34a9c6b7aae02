"""Index arithmetic of the operators around the convolutions (csrc/layers_index.h), compiled for the CPU, at sizes beyond what a test can run
and for reads that a test on the GPU must not make."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_05908_amd", "csrc")


def compiled(folder, body):
    """A program on the header whose body reads lines of numbers and prints one line for each."""
    (folder / "main.cpp").write_text("#define __host__\n#define __device__\n#include \"layers_index.h\"\n#include <cstdio>\nusing namespace fftconv::lay;\n"
                                     "int main()\n{\n" + body + "\n}\n")
    exe = str(folder / "main")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, "-o", exe,
                    str(folder / "main.cpp")], check=True)

    def ask(lines):
        text = "".join(" ".join(str(x) for x in l) + "\n" for l in lines)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(int(x) for x in l.split()) for l in out if l]

    return ask


def test_reads_of_a_gradient_end_inside_it(tmp_path):
    """dy (b, n, o), every half run that is read without a look at its end: the last sample's last piece of 8 channels ends inside the tensor. No
    more half runs than that are read the slower way, but for one a sequence."""
    ask = compiled(tmp_path, 'long long n0, n, o, t; while (std::scanf("%lld %lld %lld %lld", &n0, &n, &o, &t) == 4) std::printf("%d\\n", '
                             '(int)whole_half_run(n0, n, o, t != 0));')
    asked = [(n0, n, o, t) for t in (0, 1) for o in list(range(1, 34)) + [1001, 4097, 1 << 22] for n in list(range(1, 330)) + [(1 << 22) - 1, 1 << 22]
             for n0 in sorted({*range(0, min(n, 330), 64), max(0, (n - 1) // 64 * 64 - 64), (n - 1) // 64 * 64})]
    answers = ask(asked)
    assert len(answers) == len(asked)
    plain = 0
    for (n0, n, o, t), (whole,) in zip(asked, answers):
        last = (n0 + 63) * o + (o - 1) // 8 * 8 + 8 if t else n0 + 64      # behind the last value read: of the sequence, or of a channel's samples
        assert not whole or last <= (n * o if t else n), (n0, n, o, t)
        if n0 + 64 <= n and not whole:
            plain += 1
            assert t and last > n * o, (n0, n, o, t)
    assert plain > 0


@pytest.mark.parametrize("channels,after", [(1, 6), (2, 2), (3, 1)])
def test_reads_of_a_gradient_of_few_channels(tmp_path, channels, after):
    """The last piece of 8 reaches over several samples: not read whole with so few behind it."""
    ask = compiled(tmp_path, 'long long n0, n, o; while (std::scanf("%lld %lld %lld", &n0, &n, &o) == 3) std::printf("%d\\n", (int)whole_half_run(n0, n, o, true));')
    assert ask([(0, 64 + after, channels), (64, 128 + after, channels), (0, 64 + after + 1, channels)]) == [(0,), (0,), (1,)]


@pytest.mark.parametrize("threads", [64, 256, 512])
def test_launches_of_less_than_2_32_threads(tmp_path, threads):
    """Every workgroup in one launch, in order, none with 2^32 threads; a launch that fails is the last."""
    ask = compiled(tmp_path, """
    long long n, stop;
    while (std::scanf("%%lld %%lld", &n, &stop) == 2) {
        long long next = 0, calls = 0;
        const int rc = in_pieces(n, %d, [&](int64_t first, unsigned g) -> int {
            if (first != next || g < 1 || (long long)g * %d >= 1LL << 32) return -99;
            next = first + g;
            return ++calls == stop ? -5 : 0;
        });
        std::printf("%%d %%lld %%lld\\n", rc, calls, next);
    }""" % (threads, threads))
    most = ((1 << 32) - 1) // threads
    for n in (1, 2, most - 1, most, most + 1, 2 * most, 2 * most + 1, (1 << 35) // 32, (1 << 31) - 1):
        calls = -(-n // most)
        assert ask([(n, 0), (n, 1)]) == [(0, calls, n), (-5, 1, min(n, most))]
    assert ask([(0, 0)]) == [(0, 0, 0)]
