"""Results that overlap what else a call of the recurrent layer's operators reads or writes are refused, through the C ABI, before any device is touched.

Every tensor has a stretch of addresses of its own that are never read; a case moves one of them onto, or partly onto, another. (That tensors side by side are
taken is tested where there is a device.)"""
import pytest

from paper_2311_05908_amd import fftconv

F32, F16, BF16 = 0, 1, 2
EINVAL = -1
PAGE = 1 << 20


def places(*names):
    return {name: PAGE * (i + 1) for i, name in enumerate(names)}


def refused(name, *a):
    lib = fftconv.load()
    assert getattr(lib, name)(*a) == EINVAL
    said = lib.fftconv_last_error().decode()
    assert name in said and "overlap" in said, said


STEP = places("u", "w", "v", "state", "next", "y")


def step(dtype=F32, t=100, **moved):
    p = {**STEP, **moved}
    refused("fftconv_gated_step", p["u"], p["w"], p["v"], p["state"], p["next"], p["y"], t, 0, dtype, None)


@pytest.mark.parametrize("name", ["u", "w", "v", "state", "next"])
@pytest.mark.parametrize("dtype,size", [(F32, 4), (BF16, 2)])
def test_step(name, dtype, size):
    """100 channels: the last value of one is the first of the other, either way round, or they begin together."""
    for result, bytes_of in (("next", 400), ("y", 100 * size)):
        if name == result:
            continue
        other = 400 if name in ("state", "next") else 100 * size
        step(dtype, **{result: STEP[name] + other - 4})
        step(dtype, **{result: STEP[name] - bytes_of + 4})
        if (result, name) != ("next", "state"):
            step(dtype, **{result: STEP[name]})


def test_step_in_place():
    """next is state itself, and meets another tensor all the same."""
    for name in ("u", "w", "v", "y"):
        step(next=STEP["state"], **{name: STEP["state"]})
        step(next=STEP["state"], **{name: STEP["state"] + 396})
