"""What ptq_prompt_attention refuses, seen on the host (nothing reaches a launch)."""
import os

import pytest
import torch

import paper_2601_19675_amd as ptq

OK, ARG, SHAPE, DTYPE = 0, 1, 2, 3
P = 0x1000   # aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ptq.lib_path()):
        from paper_2601_19675_amd import build
        build.build(verbose=False)
    return ptq.load_library()


def test_prompt_attention(lib):
    ok = dict(Q=P, qt=256, qh=64, K=2 * P, kt=128, kh=64, V=3 * P, vt=128, vh=64, dt=1, t=10, hq=4, hkv=2, d=64, cu=P, b=2, max_n=7, scale=0.125,
              causal=1, window=0, O=4 * P, ot=256, oh=64, stream=None)

    def call(**kw):
        assert set(kw) <= set(ok), kw
        return lib.ptq_prompt_attention(*[{**ok, **kw}[k] for k in ok])

    assert call(t=0, max_n=0) == OK and call(b=0) == OK and call(max_n=0) == OK
    assert call(dt=0) == DTYPE and call(dt=2) == DTYPE
    for scale in (float("nan"), float("inf"), 2.1e38, -2.1e38):
        assert call(scale=scale) == ARG
    assert call(window=-1) == ARG
    assert call(d=0) == SHAPE and call(d=24) == SHAPE and call(d=272) == SHAPE and call(hkv=0) == SHAPE and call(hkv=32768, hq=32768) == SHAPE
    assert call(hq=3) == SHAPE and call(hq=0) == SHAPE and call(hq=65536) == SHAPE and call(b=65536) == SHAPE and call(b=-1) == SHAPE
    assert call(t=-1) == SHAPE and call(t=2 ** 24 + 1) == SHAPE and call(max_n=11) == SHAPE and call(max_n=-1) == SHAPE
    assert call(t=2 ** 24, max_n=2 ** 24, hq=18) == SHAPE     # rows of a key head
    for name in ("qt", "qh", "kt", "kh", "vt", "vh", "ot", "oh"):
        assert call(**{name: -1}) == SHAPE
    for name in ("Q", "K", "V", "O", "cu"):
        assert call(**{name: None}) == ARG
    assert call(O=2 * P) == ARG and call(O=3 * P) == ARG and call(O=P, ot=512) == ARG and call(O=P, oh=128) == ARG


def test_python_call_refuses_tensors_that_do_not_fit():
    x, cu = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        ptq.ptq_prompt_attention(x, x, x, cu, 2, 1.0, x)
    with pytest.raises(TypeError):
        ptq.ptq_prompt_attention(x.float().numpy(), x, x, cu, 2, 1.0, x)
