"""Results that overlap what else a call of the recurrent layer's operators reads or writes are refused, through the C ABI, before any device is touched.

Every tensor has a stretch of addresses of its own that are never read; a case moves one of them onto, or partly onto, another. (That tensors side by side are
taken is tested where there is a device.)"""
import ctypes

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


SCAN = places("u", "w", "v", "state", "lengths", "y", "last", "kept", "ws")
BACK = places("dy", "u", "w", "v", "kept", "dlast", "lengths", "du", "dw", "dv", "dstate", "ws")
B, C, N = 2, 3, 5000          # rows in segments, so that there is a workspace


def bytes_of(name, size):
    if name == "ws":
        return fftconv.load().fftconv_workspace_bytes_gated_scan(B, C, N, F32)
    return {"state": 4 * B * C, "last": 4 * B * C, "dlast": 4 * B * C, "dstate": 4 * B * C, "lengths": 4 * B, "kept": 4 * B * C * 10}.get(name, size * B * C * N)


def scan(dtype, **moved):
    p = {**SCAN, **moved}
    refused("fftconv_gated_scan", *(p[k] for k in ("u", "w", "v", "state", "lengths", "y", "last", "kept")), B, C, N, 0, dtype, p["ws"], None)


def back(dtype, **moved):
    p = {**BACK, **moved}
    refused("fftconv_gated_scan_backward", *(p[k] for k in ("dy", "u", "w", "v", "kept", "dlast", "lengths", "du", "dw", "dv", "dstate")), B, C, N, 1, dtype, p["ws"], None)


@pytest.mark.parametrize("dtype,size", [(F32, 4), (F16, 2)])
@pytest.mark.parametrize("call,all_of,results", [(scan, SCAN, ("y", "last", "kept", "ws")), (back, BACK, ("du", "dw", "dv", "dstate", "ws"))])
def test_scans(call, all_of, results, dtype, size):
    """Every result and the workspace against every other tensor: together, the first 8 bytes on its last, its last on the first. Among them last on state (dstate on
    dlast), which workgroups of a row's other segments may still have to read."""
    for result in results:
        for name in all_of:
            if name != result:
                for at in (all_of[name], all_of[name] + bytes_of(name, size) - 8, all_of[name] - bytes_of(result, size) + 8):
                    call(dtype, **{result: at - at % 8 if result == "ws" else at})


def test_scans_without_what_may_be_missing():
    """What is not there meets nothing; what is there does."""
    none = dict(v=None, state=None, lengths=None, last=None, kept=None)
    scan(F32, **none, y=SCAN["u"])
    scan(BF16, **{**none, "kept": SCAN["w"]})
    back(F32, v=None, dv=None, dlast=None, lengths=None, dstate=None, du=BACK["dy"])
    back(F16, v=None, dv=None, lengths=None, dstate=BACK["dlast"])


CLIP = places("a", "b", "out a", "out b", "given", "norm", "ws")


def clip(out=True, types=(F32, BF16), types_out=(F32, F32), counts=(100, 30), **moved):
    p = {**CLIP, "given": None, "norm": None, **moved}
    i64, ints = lambda *v: (ctypes.c_int64 * len(v))(*v), lambda *v: (ctypes.c_int * len(v))(*v)
    refused("fftconv_clip_grads", i64(p["a"], p["b"]), i64(p["out a"], p["out b"]) if out else None, i64(*counts), ints(*types), ints(*types_out), 2, 1.0, 1e-6,
            p["given"], p["norm"], p["ws"], None)


def test_a_norm_that_is_given_in_what_is_written():
    """100 values of fp32 and 30 of bf16 into fp32: every workgroup reads the norm while others write."""
    for name, size in (("out a", 400), ("out b", 120)):
        for at in (0, 4, size // 2, size - 4):
            clip(given=CLIP[name] + at, ws=None)
    for at in (0, 396):                                       # in place
        clip(given=CLIP["a"] + at, ws=None, **{"out a": CLIP["a"]})


def test_a_norm_that_is_written():
    """On a gradient, a result or the workspace, with clipping and without."""
    for name, size in (("a", 400), ("b", 60), ("out a", 400), ("out b", 120)):
        for at in (0, size - 4):
            clip(norm=CLIP[name] + at)
            if not name.startswith("out"):
                clip(norm=CLIP[name] + at, out=False)
    clip(norm=CLIP["ws"])
    clip(norm=CLIP["ws"], out=False)
    clip(norm=CLIP["out a"], given=CLIP["given"], ws=None)


def test_a_workspace_on_tensors():
    need = fftconv.load().fftconv_workspace_bytes_clip_grads((ctypes.c_int64 * 2)(100, 30), 2)
    assert need >= 16
    for name, size in (("a", 400), ("b", 60), ("out a", 400), ("out b", 120)):
        for at in (0, size // 8 * 8 - 8, 8 - need):
            clip(ws=CLIP[name] + at)
            if not name.startswith("out"):
                clip(ws=CLIP[name] + at, out=False)
