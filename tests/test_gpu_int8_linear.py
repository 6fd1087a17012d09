"""The 8-bit product against its float64 oracle: few tokens, both tile sizes, split sums, rests of every length."""
import numpy as np
import pytest
import torch

import paper_2601_19675_amd as ptq
from oracle import attention_oracle as orc

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def tensors(t, m, n, seed, pad=0, scale=30.0):
    g = np.random.default_rng(seed)
    A, W = (np.clip(np.rint(scale * g.standard_normal(s)), -128, 127).astype(np.int8) for s in ((t, n), (m, n)))
    asc, wsc = np.exp(g.standard_normal(t)).astype(np.float32), (0.01 * np.exp(g.standard_normal(m))).astype(np.float32)
    bias = g.standard_normal(m).astype(np.float32)

    def rows(x):
        y = torch.full((x.shape[0], n + pad), 77, dtype=torch.int8, device="cuda")
        y[:, :n] = torch.tensor(x)
        return y[:, :n]
    return (A, asc, W, wsc, bias), (rows(A), torch.tensor(asc, device="cuda"), rows(W), torch.tensor(wsc, device="cuda"),
                                    torch.tensor(bias, device="cuda"))


def check(t, m, n, dtype, seed, with_bias=True, pad=0, pad_out=0, exact_on_gpu=False):
    host, dev = tensors(t, m, n, seed, pad)
    A, asc, W, wsc, bias = host
    O = torch.full((t + 1, m + pad_out), 5.0, dtype=dtype, device="cuda")
    ws = None
    need = ptq.ptq_workspace_bytes(ptq.OP_INT8_LINEAR, m, n, t)
    if need:
        ws = torch.full((need + 256,), 0xEE, dtype=torch.uint8, device="cuda")   # what was there does not matter
    ptq.ptq_int8_linear(dev[0], dev[1], dev[2], dev[3], O[:t, :m], bias=dev[4] if with_bias else None, ws=None if ws is None else ws[:need])
    torch.cuda.synchronize()
    assert (O[t] == 5.0).all() and (O[:, m:] == 5.0).all() and (ws is None or (ws[need:] == 0xEE).all())
    if exact_on_gpu:   # whole products of these sizes are quick in float64 there
        sums = dev[0].double() @ dev[2].double().T
        want = sums * dev[1].double()[:, None] * dev[3].double() + (dev[4].double() if with_bias else 0.0)
        size = (sums * dev[1].double()[:, None] * dev[3].double()).abs() + (dev[4].double().abs() if with_bias else 0.0)
        got, want, size = O[:t, :m].double().cpu().numpy(), want.cpu().numpy(), size.cpu().numpy()
    else:
        want = orc.int8_linear(A, asc, W, wsc, bias if with_bias else None)
        size = np.abs(orc.int8_linear(A, asc, W, wsc)) + (np.abs(bias).astype(np.float64) if with_bias else 0.0)
        got = O[:t, :m].double().cpu().numpy()
    # to float32, two scales, one addition: a rounding each of 2^-24 of at most `size`; then the one to the output's type
    assert np.all(np.abs(got - want) <= 4.1 * 2.0 ** -24 * size + (HALF[dtype] * 1.01 * np.abs(want) if dtype == torch.bfloat16 else 0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [1, 2, 15, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("m,n", [(1, 16), (17, 64), (64, 80), (100, 1008), (33, 4096)])
def test_few_tokens(dtype, t, m, n):
    check(t, m, n, dtype, seed=t * 31 + m + n, with_bias=t % 2 == 0, pad=16 * (t % 3), pad_out=t % 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t,m,n", [(65, 1, 16), (70, 129, 48), (128, 128, 64), (129, 127, 128), (200, 65, 192), (65, 300, 208), (130, 131, 320),
                                   (257, 255, 1040), (66, 70, 4096), (300, 130, 2000)])
def test_tiles(dtype, t, m, n):
    check(t, m, n, dtype, seed=t + m + n, with_bias=m % 2 == 1, pad=16 * (t % 2), pad_out=t % 4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t,m,n", [(3329, 3585, 80), (4000, 3333, 336), (257, 49000, 64), (12200, 1025, 16)])
def test_large_tiles(dtype, t, m, n):
    check(t, m, n, dtype, seed=t + m + n, with_bias=m % 2 == 1, exact_on_gpu=True)


@pytest.mark.parametrize("t", [4, 200])
def test_largest_sums(t):
    # -128 * -128 over 131056 columns: the largest sum that fits
    n, m = 131056, 20
    A = torch.full((t, n), -128, dtype=torch.int8, device="cuda")
    W = torch.full((m, n), -128, dtype=torch.int8, device="cuda")
    W[1] = 127
    O = torch.zeros((t, m), device="cuda")
    ptq.ptq_int8_linear(A, torch.ones(t, device="cuda"), W, torch.ones(m, device="cuda"), O)
    torch.cuda.synchronize()
    assert (O[:, 0] == float(np.float32(16384 * n))).all() and (O[:, 1] == float(np.float32(-128 * 127 * n))).all()


def test_scales_that_are_not_finite_stay_in_their_row_and_column():
    host, dev = tensors(80, 70, 64, 9)
    dev[1][3], dev[3][5] = float("nan"), float("inf")
    O = torch.zeros((80, 70), device="cuda")
    ptq.ptq_int8_linear(dev[0], dev[1], dev[2], dev[3], O)
    bad = torch.zeros((80, 70), dtype=torch.bool, device="cuda")
    bad[3], bad[:, 5] = True, True
    assert torch.equal(~torch.isfinite(O), bad)


@pytest.mark.parametrize("t,m,n", [(3, 512, 1024), (150, 512, 4096), (3400, 3600, 128)])
def test_its_stream_and_graph(t, m, n):
    _, dev = tensors(t, m, n, 11)
    want = torch.zeros((t, m), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, ptq.ptq_workspace_bytes(ptq.OP_INT8_LINEAR, m, n, t)), dtype=torch.uint8, device="cuda")
    ptq.ptq_int8_linear(*dev[:4], want, bias=dev[4], ws=ws)
    torch.cuda.synchronize()
    got = torch.zeros_like(want)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ptq.ptq_int8_linear(*dev[:4], got, bias=dev[4], ws=ws)
    s.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ptq.ptq_int8_linear(*dev[:4], got, bias=dev[4], ws=ws)
    for _ in range(3):
        got.zero_()
        ws.fill_(0xAB)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
