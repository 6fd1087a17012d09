"""What the rotation's and the page copy's calls refuse, and the frequencies, seen on the host (nothing reaches a launch)."""
import math
import os

import pytest
import torch

import paper_2601_19675_amd as ptq

OK, ARG, SHAPE, DTYPE = 0, 1, 2, 3
P = 0x1000   # aligned, never dereferenced
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ptq.lib_path()):
        from paper_2601_19675_amd import build
        build.build(verbose=False)
    return ptq.load_library()


def caller(fn, **defaults):
    def call(**kw):
        assert set(kw) <= set(defaults), kw
        return fn(*[{**defaults, **kw}[k] for k in defaults])
    return call


def test_rotary(lib):
    call = caller(lib.ptq_rotary, X=P, xt=256, xh=64, dt=1, t=4, heads=4, d=64, positions=P, freq=P, rot=64, scale=1.0, interleaved=0, Y=2 * P,
                  yt=256, yh=64, stream=None)
    assert call(t=0) == OK and call(heads=0) == OK
    assert call(dt=2) == DTYPE and call(dt=-1) == DTYPE
    assert call(scale=NAN) == ARG and call(scale=INF) == ARG
    assert call(rot=0) == SHAPE and call(rot=66) == SHAPE and call(rot=31) == SHAPE and call(rot=-2) == SHAPE
    assert call(d=65537, rot=64) == SHAPE and call(d=0) == SHAPE and call(heads=-1) == SHAPE and call(heads=65536) == SHAPE
    assert call(t=-1) == SHAPE and call(t=2 ** 30) == SHAPE
    for name in ("xt", "xh", "yt", "yh"):
        assert call(**{name: -1}) == SHAPE
    for name in ("X", "Y", "positions", "freq"):
        assert call(**{name: None}) == ARG
    assert call(Y=P, yt=512) == ARG and call(Y=P, yh=128) == ARG     # in place, but elsewhere


def test_rotary_kv_cache_write(lib):
    call = caller(lib.ptq_rotary_kv_cache_write, Q=P, qt=512, qh=64, hq=8, K=2 * P, kt=256, kh=64, V=3 * P, vt=256, vh=64, dt=1, t=4, hkv=4, d=64,
                  positions=P, freq=P, rot=64, scale=1.0, interleaved=0, slots=P, bits=8, codes=P, scales=P, zeros=P, pages=8, page=16, O=P, ot=512,
                  oh=64, stream=None)
    assert call(t=0) == OK
    assert call(dt=2) == DTYPE and call(dt=-1) == DTYPE
    assert call(bits=3) == ARG and call(scale=NAN) == ARG and call(codes=P + 8) == ARG
    assert call(rot=8) == SHAPE and call(rot=24) == SHAPE and call(rot=80) == SHAPE and call(rot=0) == SHAPE
    assert call(d=72) == SHAPE and call(d=272) == SHAPE and call(hq=0) == SHAPE and call(hq=65536) == SHAPE and call(hkv=0) == SHAPE
    assert call(page=24) == SHAPE and call(pages=-1) == SHAPE and call(t=-1) == SHAPE
    for name in ("qt", "qh", "kt", "kh", "vt", "vh", "ot", "oh"):
        assert call(**{name: -1}) == SHAPE
    for name in ("Q", "K", "V", "positions", "freq", "slots", "codes", "scales", "zeros", "O"):
        assert call(**{name: None}) == ARG
    assert call(ot=1024) == ARG and call(O=2 * P) == ARG and call(O=3 * P) == ARG


def test_copy_pages(lib):
    call = caller(lib.ptq_kv_cache_copy_pages, fc=P, fs=P, fz=P, fp=8, codes=P, scales=P, zeros=P, pages=4, page=16, hkv=4, row=64, source=P,
                  target=P, n=3, stream=None)
    assert call(n=0) == OK and call(fp=0) == OK and call(pages=0) == OK
    assert call(row=0) == SHAPE and call(row=12) == SHAPE and call(row=264) == SHAPE and call(n=-1) == SHAPE and call(n=2 ** 31) == SHAPE
    assert call(page=24) == SHAPE and call(page=512) == SHAPE and call(hkv=0) == SHAPE and call(fp=-1) == SHAPE and call(pages=2 ** 31 // 16) == SHAPE
    for name in ("fc", "fs", "fz", "codes", "scales", "zeros", "source", "target"):
        assert call(**{name: None}) == ARG
    assert call(fc=P + 8) == ARG and call(codes=P + 8) == ARG


def test_frequencies():
    f = ptq.ptq_rotary_frequencies(128)
    want = [10000.0 ** (-2 * j / 128) for j in range(64)]
    close = lambda a, b: all(abs(x - y) <= 1e-14 * abs(y) for x, y in zip(a.tolist(), b)) and len(a) == len(b)
    assert f.dtype == torch.float64 and close(f, want)
    assert close(ptq.ptq_rotary_frequencies(128, 10000.0, ptq.PTQ_ROTARY_LINEAR, 4.0), [x / 4 for x in want])
    g = ptq.ptq_rotary_frequencies(128, 10000.0, ptq.PTQ_ROTARY_BASE, 4.0)
    assert close(g, [(10000.0 * 4 ** (128 / 126)) ** (-2 * j / 128) for j in range(64)])
    assert g[0] == 1 and abs(g[-1] * 4 / want[-1] - 1) < 1e-12
    g = ptq.ptq_rotary_frequencies(128, 500000.0, ptq.PTQ_ROTARY_TURNS, 8.0, 8192.0, 1.0, 4.0)
    for j, x in enumerate(g.tolist()):
        f = 500000.0 ** (-2 * j / 128)
        turns = 8192 * f / (2 * math.pi)
        k = min(1, max(0, (turns - 1) / 3))
        assert abs(x - f * (k + (1 - k) / 8)) <= 1e-14 * f
        assert turns < 4 or x == f
    assert ptq.ptq_rotary_frequencies(2).tolist() == [1.0]


def test_frequencies_that_are_refused(lib):
    room = torch.zeros(8, dtype=torch.float64)
    ok = dict(freq=room.data_ptr(), rot=16, base=1e4, scaling=3, factor=8.0, context=8192.0, slow=1.0, fast=4.0)
    call = caller(lib.ptq_rotary_frequencies, **ok)
    assert call() == OK and call(scaling=0, factor=-1.0, context=NAN) == OK
    assert call(rot=0) == SHAPE and call(rot=15) == SHAPE and call(rot=2, scaling=2) == SHAPE and call(rot=65538) == SHAPE
    for kw in (dict(freq=None), dict(base=0.0), dict(base=INF), dict(scaling=4), dict(scaling=-1), dict(factor=0.0), dict(factor=NAN),
               dict(context=0.0), dict(fast=1.0), dict(slow=NAN), dict(fast=INF)):
        assert call(**kw) == ARG, kw
    with pytest.raises(ptq.PtqError):
        ptq.ptq_rotary_frequencies(7)


def test_python_calls_refuse_tensors_that_do_not_fit():
    x, i, f = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="device tensors"):
        ptq.ptq_rotary(x, i, f, x)
    with pytest.raises(TypeError):
        ptq.ptq_rotary(x.numpy(), i, f, x)
    with pytest.raises(ValueError, match="device tensors"):
        ptq.ptq_rotary_kv_cache_write(x, x, x, i, f, i, 8, x, x, x, x)
    with pytest.raises(ValueError, match="device tensors"):
        ptq.ptq_kv_cache_copy_pages(x, x, x, i, x, x, x, i)
