"""What the calls of the 8-bit attention path refuse, seen on the host (none of these reaches a launch)."""
import os

import pytest

import paper_2601_19675_amd as ptq

OK, ARG, SHAPE, DTYPE, WORKSPACE = 0, 1, 2, 3, 4
P = 0x1000   # aligned, never dereferenced


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


def test_norm(lib):
    call = caller(lib.ptq_rmsnorm_quantize, X=P, dt=1, ldx=64, t=4, n=64, residual=P, ldr=64, out=P, ldo=64, gamma=P, eps=1e-5,
                  normalize=1, codes=P, ldc=64, scales=P, stream=None)
    assert call(t=0) == OK and call(n=0) == OK
    assert call(dt=2) == DTYPE and call(dt=7) == DTYPE
    assert call(eps=-1.0) == ARG and call(eps=float("nan")) == ARG and call(eps=float("inf")) == ARG
    assert call(X=None) == ARG and call(codes=None) == ARG and call(scales=None) == ARG and call(codes=P + 8) == ARG
    assert call(residual=None) == ARG        # nowhere to take the sum from
    assert call(t=-1) == SHAPE and call(n=-1) == SHAPE and call(n=32769, ldx=40000, ldc=40000, ldr=40000, ldo=40000) == SHAPE
    assert call(ldx=63) == SHAPE and call(ldr=63) == SHAPE and call(ldo=63) == SHAPE and call(ldc=48) == SHAPE and call(ldc=72) == SHAPE


def test_cache(lib):
    write = caller(lib.ptq_kv_cache_write, K=P, kt=256, kh=64, V=P, vt=256, vh=64, dt=1, t=4, hkv=4, d=64, slots=P, bits=8, codes=P,
                   scales=P, zeros=P, pages=8, page=16, stream=None)
    read = caller(lib.ptq_kv_cache_read, codes=P, scales=P, zeros=P, pages=8, page=16, hkv=4, d=64, bits=8, table=P, ldt=2, b=2, cu=P,
                  rows=40, max_kv=20, K=P, kt=256, kh=64, V=P, vt=256, vh=64, dt=1, stream=None)
    assert write(t=0) == OK and read(b=0) == OK and read(rows=0) == OK and read(max_kv=0) == OK
    for call in (write, read):
        assert call(dt=2) == DTYPE and call(dt=-1) == DTYPE
        assert call(bits=2) == ARG and call(bits=3) == ARG and call(bits=16) == ARG
        assert call(d=0) == SHAPE and call(d=72) == SHAPE and call(d=272) == SHAPE
        assert call(hkv=0) == SHAPE and call(hkv=32768) == SHAPE
        assert call(page=0) == SHAPE and call(page=24) == SHAPE and call(page=512) == SHAPE
        assert call(pages=-1) == SHAPE and call(pages=2 ** 31 // 16) == SHAPE
        assert call(kt=-1) == SHAPE and call(vh=-1) == SHAPE
        for name in ("K", "V", "codes", "scales", "zeros"):
            assert call(**{name: None}) == ARG
        assert call(codes=P + 8) == ARG
    assert write(slots=None) == ARG and write(t=-1) == SHAPE
    assert read(table=None) == ARG and read(cu=None) == ARG and read(pages=0) == SHAPE
    assert read(b=65536) == SHAPE and read(ldt=-1) == SHAPE and read(ldt=0) == SHAPE and read(rows=-1) == SHAPE and read(max_kv=-1) == SHAPE


def test_int8_linear(lib):
    call = caller(lib.ptq_int8_linear, A=P, lda=64, asc=P, t=4, W=P, ldw=64, wsc=P, m=8, n=64, bias=None, O=P, odt=1, ldo=8, ws=None,
                  bytes=0, stream=None)
    assert call(t=0) == OK and call(m=0, ldo=0) == OK
    assert call(odt=2) == DTYPE
    assert call(n=0) == SHAPE and call(n=24) == SHAPE and call(lda=48) == SHAPE and call(lda=72) == SHAPE and call(ldw=48) == SHAPE
    assert call(n=131072, lda=131072, ldw=131072) == SHAPE and call(lda=2 ** 22 + 16) == SHAPE and call(ldw=2 ** 22 + 16) == SHAPE
    assert call(ldo=7) == SHAPE and call(t=-1) == SHAPE and call(m=-1) == SHAPE
    for name in ("A", "asc", "W", "wsc", "O"):
        assert call(**{name: None}) == ARG
    assert call(A=P + 8) == ARG and call(W=P + 4) == ARG
    need = ptq.ptq_workspace_bytes(ptq.OP_INT8_LINEAR, 1000, 11008, 100)   # a size whose sums are split
    assert need > 0
    big = dict(t=100, m=1000, n=11008, lda=11008, ldw=11008, ldo=1000)
    assert call(**big) == WORKSPACE and call(**big, ws=P, bytes=need - 1) == WORKSPACE and call(**big, ws=P + 8, bytes=need) == WORKSPACE
    assert ptq.ptq_workspace_bytes(ptq.OP_INT8_LINEAR, 4096, 4096, 1) == 0


def test_paged_attention(lib):
    call = caller(lib.ptq_paged_attention, Q=P, dt=1, qt=256, qh=64, t=4, hq=4, d=64, cu=P, b=2, max_q=3, codes=P, scales=P, zeros=P, pages=8,
                  page=16, hkv=2, bits=8, table=P, ldt=2, lens=P, max_kv=20, scale=0.125, causal=1, window=0, O=2 * P, ot=256, oh=64,
                  ws=None, bytes=0, stream=None)
    assert call(t=0, max_q=0) == OK and call(b=0) == OK and call(max_q=0) == OK
    assert call(dt=0) == DTYPE and call(dt=2) == DTYPE
    assert call(bits=2) == ARG and call(scale=float("nan")) == ARG and call(scale=float("inf")) == ARG and call(window=-1) == ARG
    assert call(d=72) == SHAPE and call(d=272) == SHAPE and call(page=24) == SHAPE and call(hkv=0) == SHAPE and call(pages=0) == SHAPE
    assert call(hq=3) == SHAPE and call(hq=0) == SHAPE and call(b=65536) == SHAPE and call(max_q=5) == SHAPE and call(max_q=-1) == SHAPE
    assert call(t=-1) == SHAPE and call(ldt=-1) == SHAPE and call(max_kv=-1) == SHAPE and call(qt=-1) == SHAPE and call(oh=-1) == SHAPE
    for name in ("Q", "O", "cu", "codes", "scales", "zeros", "table", "lens"):
        assert call(**{name: None}) == ARG
    assert call(codes=P + 8) == ARG and call(O=P) == ARG
    need = ptq.ptq_workspace_bytes(ptq.OP_PAGED_ATTENTION, 4, 64, 4, 5000)
    assert need > 0 and call(max_kv=5000) == WORKSPACE and call(max_kv=5000, ws=P, bytes=need - 1) == WORKSPACE
    assert ptq.ptq_workspace_bytes(ptq.OP_PAGED_ATTENTION, 32, 128, 3000, 16384) < 300 << 20


def test_python_calls_refuse_tensors_that_do_not_fit():
    import torch
    x, c = torch.zeros((2, 64)), torch.zeros((2, 64), dtype=torch.int8)
    with pytest.raises(ValueError, match="device tensors"):
        ptq.ptq_rmsnorm_quantize(x, c, torch.zeros(2))
    with pytest.raises(ValueError, match="device tensors"):
        ptq.ptq_int8_linear(c, torch.zeros(2), c, torch.zeros(2), torch.zeros((2, 2)))
    with pytest.raises(TypeError):
        ptq.ptq_rmsnorm_quantize(x.numpy(), c, torch.zeros(2))
    with pytest.raises(TypeError):
        ptq.ptq_kv_cache_write(None, x, c, 8, c, x, c)
