"""What ptq_paged_attention_shared refuses, seen on the host (nothing reaches a launch)."""
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


def test_paged_attention_shared(lib):
    ok = dict(Q=P, dt=1, qt=256, qh=64, t=4, hq=4, d=64, cu=P, b=2, max_q=3, codes=P, scales=P, zeros=P, pages=8, page=16, hkv=2, bits=8, table=P, ldt=2,
              lens=P, max_kv=20, groups_at=P, shared=P, groups=1, max_shared=16, scale=0.125, causal=1, O=2 * P, ot=256, oh=64, ws=None, bytes=0,
              stream=None)

    def call(**kw):
        assert set(kw) <= set(ok), kw
        return lib.ptq_paged_attention_shared(*[{**ok, **kw}[k] for k in ok])

    assert call(t=0, max_q=0) == OK and call(b=0) == OK and call(max_q=0) == OK
    assert call(dt=0) == DTYPE and call(dt=2) == DTYPE
    assert call(bits=2) == ARG and call(scale=float("nan")) == ARG and call(scale=2.1e38) == ARG
    assert call(d=72) == SHAPE and call(d=272) == SHAPE and call(page=24) == SHAPE and call(hkv=0) == SHAPE and call(pages=0) == SHAPE
    assert call(hq=3) == SHAPE and call(hq=0) == SHAPE and call(b=65536) == SHAPE and call(max_q=5) == SHAPE and call(max_q=-1) == SHAPE
    assert call(t=-1) == SHAPE and call(ldt=-1) == SHAPE and call(max_kv=-1) == SHAPE and call(qt=-1) == SHAPE and call(oh=-1) == SHAPE
    assert call(groups=-1) == SHAPE and call(groups=65536) == SHAPE and call(max_shared=-1) == SHAPE and call(t=2 ** 24, hq=32, hkv=2) == SHAPE
    for name in ("Q", "O", "cu", "codes", "scales", "zeros", "table", "lens", "groups_at", "shared"):
        assert call(**{name: None}) == ARG
    assert call(codes=P + 8) == ARG and call(O=P) == ARG
    need = ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, 4, 64, 4, 20)
    assert need > 0 and call() == WORKSPACE and call(ws=P, bytes=need - 1) == WORKSPACE and call(ws=P + 8, bytes=need) == WORKSPACE


@pytest.mark.parametrize("hq,d,t,max_kv", [(4, 64, 1, 1), (32, 128, 64, 33500), (64, 256, 3000, 16384), (16, 16, 5, 0)])
def test_the_workspace_is_enough_for_the_call_without_groups(hq, d, t, max_kv):
    shared, plain = (ptq.ptq_workspace_bytes(op, hq, d, t, max_kv) for op in (ptq.OP_SHARED_ATTENTION, ptq.OP_PAGED_ATTENTION))
    assert shared >= plain and shared % 256 == 0 and shared < 600 << 20
