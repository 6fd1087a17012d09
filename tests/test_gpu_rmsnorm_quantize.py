"""The norm into 8 bits against its float64 oracle: codes and the residual sum exactly, scales to float32's rounding."""
import numpy as np
import pytest
import torch

import paper_2601_19675_amd as ptq
from oracle import attention_oracle as orc

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def put(a, dtype, pad=0):
    """A device tensor of a's values, rows `pad` elements apart from each other."""
    x = torch.zeros((a.shape[0], a.shape[1] + pad), dtype=DT[dtype], device="cuda")
    x[:, : a.shape[1]] = torch.tensor(np.asarray(a, dtype=np.float32)).to(DT[dtype])
    return x[:, : a.shape[1]]


def run(X, dtype, residual=None, gamma=None, eps=1e-5, normalize=True, pad=0, inplace=False):
    t, n = X.shape
    x, r = put(X, dtype, pad), None if residual is None else put(residual, dtype, pad + 3)
    g = None if gamma is None else put(gamma[None], dtype)[0].contiguous()
    codes = torch.full((t, -(-n // 16) * 16 + 16), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((t,), 7.0, device="cuda")
    out = None if r is None else r if inplace else torch.zeros((t, n + 5), dtype=DT[dtype], device="cuda")[:, :n]
    ptq.ptq_rmsnorm_quantize(x, codes[:, :n], scales, gamma=g, residual=r, residual_out=out, eps=eps, normalize=normalize)
    torch.cuda.synchronize()
    assert (codes[:, n:] == 99).all()   # nothing past the row's end
    return codes[:, :n].cpu().numpy(), scales.cpu().numpy(), None if out is None else out.float().cpu().numpy()


def check(X, dtype, residual=None, gamma=None, eps=1e-5, normalize=True, **kw):
    codes, scales, out = run(X, dtype, residual, gamma, eps, normalize, **kw)
    want, ws, y = orc.rmsnorm_quantize(X, dtype, residual, gamma, eps, normalize)
    assert (codes == want).all()
    # float64 inside, rounded once: 2^-24 of the value, doubled for the sums' order and the definition's own rounding
    assert np.array_equal(np.isnan(scales), np.isnan(ws))
    ok = ~np.isnan(ws)
    assert np.all(np.abs(scales[ok] - ws[ok]) <= 2.0 ** -23 * np.abs(ws[ok]) + 2.0 ** -149)
    if out is not None:
        assert np.array_equal(out, y.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t,n", [(1, 1), (3, 7), (2, 8), (5, 64), (4, 513), (3, 1024), (6, 2048), (2, 2049), (3, 4096), (2, 4097),
                                 (2, 8200), (1, 11008), (2, 12289), (2, 16384), (1, 16385), (2, 32768)])
def test_sizes(dtype, t, n):
    g = np.random.default_rng(t * 100003 + n)
    X = orc.store(g.standard_normal((t, n)) * np.exp(g.standard_normal(n)), dtype)
    R = orc.store(3 * g.standard_normal((t, n)), dtype)
    G = orc.store(1 + 0.2 * g.standard_normal(n), dtype)
    check(X, dtype)
    check(X, dtype, residual=R, gamma=G, pad=1)
    check(X, dtype, residual=R, gamma=G, inplace=True)
    check(X, dtype, gamma=G, normalize=False, pad=5)
    check(X, dtype, residual=R, normalize=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_borders_between_codes(dtype):
    # rows whose values are exact middles of two codes: 254 u = (2 k + 1) A with A = 254
    k = np.arange(-126, 126)
    X = np.concatenate(([254.0], (2 * k + 1).astype(np.float64)))[None]
    X = np.concatenate((X, X / 8, -X * 2.0 ** 60, X * 2.0 ** -100, X * 2.0 ** -120))
    check(orc.store(X, dtype), dtype, normalize=False)
    if dtype == "f32":   # and their neighbours
        F = X.astype(np.float32)
        check(np.concatenate((F[:, :1], np.nextafter(F[:, 1:], np.float32(np.inf), dtype=np.float32)), 1), dtype, normalize=False)
        check(np.concatenate((F[:, :1], np.nextafter(F[:, 1:], np.float32(-np.inf), dtype=np.float32)), 1), dtype, normalize=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_rows(dtype):
    big, tiny = float(orc.store([3e38], dtype)[0]), 2.0 ** -133
    X = np.zeros((9, 70))
    X[1, 3] = -tiny                       # one value, the smallest kind
    X[2] = big                            # squares beyond float32
    X[3, :] = np.linspace(-1, 1, 70) * big
    X[4, 69] = np.inf
    X[5, 0] = np.nan
    X[6, 17] = -np.inf
    X[7] = 2.0 ** -126
    X[8] = np.arange(70) * tiny
    X = orc.store(X, dtype)
    X[4, 69], X[5, 0], X[6, 17] = np.inf, np.nan, -np.inf
    check(X, dtype)
    check(X, dtype, normalize=False)
    # the sum overflows
    R = np.zeros_like(X)
    R[2] = big
    with np.errstate(over="ignore", invalid="ignore"):
        codes, scales, out = run(X, dtype, residual=R)
    assert np.isnan(scales[2]) and not codes[2].any() and np.isinf(out[2]).all()


def test_nothing_to_do():
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    ptq.ptq_rmsnorm_quantize(x, torch.zeros((0, 64), dtype=torch.int8, device="cuda"), torch.zeros((0,), device="cuda"))


def test_its_stream():
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((300, 512), generator=g, device="cuda")
    want, ws = torch.zeros((300, 512), dtype=torch.int8, device="cuda"), torch.zeros((300,), device="cuda")
    ptq.ptq_rmsnorm_quantize(x, want, ws)
    torch.cuda.synchronize()
    got, gs = torch.zeros_like(want), torch.zeros_like(ws)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = x * 1.0
        ptq.ptq_rmsnorm_quantize(y, got, gs)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(gs, ws)
