"""The attention half of a decoder layer out of the library's calls against the same layer in float64, without tokens, keys and values
being rounded.

Bound: a token's, key's or value's code is off by half a step, 1 / 254 of the row's largest value (8 bits) or 1 / 510 of its range;
random rows of 64 to 512 channels have their largest value within 4.5 root mean squares, so each of the three roundings (normed tokens, cache,
attended tokens) moves a row by at most 4.5 / 254 of its length, and as much again where scores move weights; the weights that are
compared against are the rounded ones.  Four times that, 7 %, and 16 / 255 in place of it for the cache in 4 bits (9 / 30 of a root
mean square for a half step, uniformly spread: 3 ** -0.5 of it, twice), 40 %."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("decoder_attention", os.path.join(os.path.dirname(__file__), "..", "examples", "decoder_attention.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)

SIZES = dict(hidden=512, heads=8, kv_heads=2, d=64, page=16, sequences=3, max_kv=400, max_tokens=700)
BOUND = {8: 0.07, 4: 0.40}


def plain(half, gamma, x, residual):
    """One sequence's tokens from the first on: float64 on the CPU, the half's own 8-bit weights."""
    r = (x.double() + (0 if residual is None else residual.double())).cpu()
    n = r * (r.pow(2).mean(dim=1, keepdim=True) + half.eps).rsqrt() * gamma.double().cpu()
    w = lambda c, s: c.double().cpu() * s.double().cpu()[:, None]
    qkv = n @ w(half.wqkv, half.wqkv_scales).T
    t, h, g, d = x.shape[0], half.heads, half.kv_heads, half.d
    q, k, v = (p.reshape(t, -1, d) for p in qkv.split([h * d, g * d, g * d], dim=1))
    out = torch.empty(t, h, d, dtype=torch.float64)
    see = torch.ones(t, t).tril().bool()
    for i in range(h):
        s = (q[:, i] @ k[:, i // (h // g)].T * d ** -0.5).masked_fill(~see, float("-inf"))
        out[:, i] = s.softmax(dim=1) @ v[:, i // (h // g)]
    return out.reshape(t, h * d) @ w(half.wo, half.wo_scales).T, r


@pytest.mark.parametrize("bits", [8, 4])
def test_prompts_in_chunks_then_single_tokens(bits):
    half, (gamma, _, _) = example.make_half(bits=bits, seed=bits, **SIZES)
    g = torch.Generator(device="cuda").manual_seed(7)
    lengths, tail = [300, 37, 160], 5   # tokens of each sequence, the last `tail` one at a time
    xs = [torch.randn(n, 512, device="cuda", generator=g).bfloat16() for n in lengths]
    rs = [torch.randn(n, 512, device="cuda", generator=g).bfloat16() for n in lengths]
    got = [[] for _ in lengths]
    sums = [[] for _ in lengths]
    done = [0] * 3
    steps = [[120, 20, 100], [175, 12, 55]] + [[1, 1, 1]] * tail
    for step in steps:
        cut = lambda a: torch.cat([a[s][done[s]:done[s] + n] for s, n in enumerate(step)])
        out, total = half(cut(xs), cut(rs), half.cache.extend(step))
        for s, (o, t) in enumerate(zip(out.clone().split(step), total.clone().split(step))):
            got[s].append(o)
            sums[s].append(t)
            done[s] += step[s]
    assert done == lengths == half.cache.lens
    for s in range(3):
        want, r = plain(half, gamma, xs[s], rs[s])
        o, t = torch.cat(got[s]).double().cpu(), torch.cat(sums[s]).double().cpu()
        assert (t - r).abs().max() <= r.abs().max() * 2 ** -8    # one rounding to bfloat16
        err = ((o - want).norm() / want.norm()).item()
        assert err < BOUND[bits], err
        err = ((o - want)[-tail:].norm() / want[-tail:].norm()).item()
        assert err < BOUND[bits], err


def test_single_tokens_from_a_graph():
    half, _ = example.make_half(seed=3, **SIZES)
    g = torch.Generator(device="cuda").manual_seed(8)
    prompt = torch.randn(600, 512, device="cuda", generator=g).bfloat16()
    half(prompt, None, half.cache.extend([300, 200, 100]))
    x, r = (torch.randn(3, 512, device="cuda", generator=g).bfloat16() for _ in range(2))
    at = half.cache.extend([1, 1, 1])
    half(x, r, at)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        half(x, r, at)
    for i in range(20):   # past the end of a page
        x.copy_(torch.randn(3, 512, device="cuda", generator=g).bfloat16())
        now = half.cache.extend([1, 1, 1])
        at["slots"].copy_(now["slots"])
        at["kv_lens"].copy_(now["kv_lens"])
        graph.replay()
        out = half.out[:3].clone()
        half(x, r, now)   # the same tokens into the same slots
        assert torch.equal(half.out[:3], out), i
    K, V, cu = half.cache.read(half.kv_heads, half.d)
    assert cu == [0, 321, 542, 663] and bool(torch.isfinite(K).all() & torch.isfinite(V).all())


def test_command_runs(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["decoder_attention.py", "--sequences", "2", "--context", "96", "--chunk", "64", "--new", "4", "--bits", "4"])
    example.main()
    assert "finite True" in capsys.readouterr().out
