"""Rotary positions, whole prompts, forks and the attention behind what they share, run together as the example does, against the layer in
float64 without any rounding.  Bound: as in test_gpu_decoder_attention_example.py; whole prompts round less."""
import pytest
import torch

from oracle import attention_oracle as oracle
from test_gpu_decoder_attention_example import BOUND, example

pytestmark = pytest.mark.gpu
SIZES = dict(hidden=512, heads=8, kv_heads=2, d=64, page=16, max_kv=500, max_tokens=700, rotary=True, whole_prompts=True)


def plain(half, gamma, x, residual):
    """One sequence's tokens from the first on: float64 on the CPU, the half's own 8-bit weights."""
    r = (x.double() + (0 if residual is None else residual.double())).cpu()
    n = r * (r.pow(2).mean(dim=1, keepdim=True) + half.eps).rsqrt() * gamma.double().cpu()
    w = lambda c, s: c.double().cpu() * s.double().cpu()[:, None]
    qkv = n @ w(half.wqkv, half.wqkv_scales).T
    t, h, g, d = x.shape[0], half.heads, half.kv_heads, half.d
    q, k, v = (p.reshape(t, -1, d) for p in qkv.split([h * d, g * d, g * d], dim=1))
    q, k = (torch.from_numpy(oracle.rotary(p.numpy(), range(t), half.freq.cpu().numpy())) for p in (q, k))
    out = torch.empty(t, h, d, dtype=torch.float64)
    see = torch.ones(t, t).tril().bool()
    for i in range(h):
        s = (q[:, i] @ k[:, i // (h // g)].T * d ** -0.5).masked_fill(~see, float("-inf"))
        out[:, i] = s.softmax(dim=1) @ v[:, i // (h // g)]
    return out.reshape(t, h * d) @ w(half.wo, half.wo_scales).T


@pytest.mark.parametrize("bits", [8, 4])
def test_answers_behind_shared_prompts(bits):
    half, (gamma, _, _) = example.make_half(bits=bits, seed=bits, sequences=7, **SIZES)
    cache, g = half.cache, torch.Generator(device="cuda").manual_seed(5)
    rand = lambda n: torch.randn(n, 512, device="cuda", generator=g).bfloat16()
    prompts = {0: rand(300), 3: rand(37), 4: rand(210)}
    outs = {}
    # prompts in one piece, two of them at a time, then one by itself
    out, _ = half(torch.cat([prompts[0], prompts[4]]), None, cache.extend([300, 0, 0, 0, 210, 0, 0]))
    outs[0], outs[4] = out[:300].clone(), out[300:].clone()
    out, _ = half(prompts[3], None, cache.extend([0, 0, 0, 37, 0, 0, 0]))
    outs[3] = out.clone()
    cache.fork([[0, 1, 2], [4, 5, 6]])
    parent = [0, 0, 0, 3, 4, 4, 4]
    # full pages are shared: 18 of 300 tokens, 13 of 210; the page after them is everybody's own
    assert torch.equal(cache.table[1, :18], cache.table[0, :18]) and cache.table[1, 18] != cache.table[0, 18] != cache.table[2, 18]
    assert torch.equal(cache.table[6, :13], cache.table[4, :13]) and sum(1 for u in cache.users if u) == 19 + 2 + 3 + 14 + 2
    tails = [[] for _ in range(7)]
    got = [[] for _ in range(7)]
    x = rand(7)
    at = cache.extend([1] * 7)
    graph = None
    for step in range(6):
        if step:
            x.copy_(rand(7))
            now = cache.extend([1] * 7)
            for name in ("slots", "kv_lens", "positions"):
                at[name].copy_(now[name])
        if step < 2:
            half(x, None, at)
        elif graph is None:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                half(x, None, at)
            graph.replay()
        else:
            graph.replay()
        for s in range(7):
            tails[s].append(x[s:s + 1].clone())
            got[s].append(half.out[s:s + 1].clone())
    for s in range(7):
        want = plain(half, gamma, torch.cat([prompts[parent[s]]] + tails[s]), None)
        if s == parent[s]:
            n = outs[s].shape[0]
            o = outs[s].double().cpu()
            assert ((o - want[:n]).norm() / want[:n].norm()).item() < BOUND[8]      # the prompt's own keys and values are not rounded to codes
        o = torch.cat(got[s]).double().cpu()
        err = ((o - want[-6:]).norm() / want[-6:].norm()).item()
        assert err < BOUND[bits], (s, err)
    # the same token once more, every context gone through by itself
    mine = half.out[:7].clone()
    cache.max_shared, shared = 0, cache.max_shared
    half(x, None, at)
    assert ((half.out[:7].double() - mine.double()).norm() / mine.double().norm()).item() < 2.0 ** -5
    cache.max_shared = shared
    # a family's parent goes, the others stay; the pages in use move together; what is read back stays what it was
    K, V, cu = cache.read(half.kv_heads, half.d)
    cache.release(4)
    cache.release(1)
    used = sum(1 for u in cache.users if u)
    cache.compact()
    assert all(u > 0 for u in cache.users[:used]) and not any(cache.users[used:]) and int(cache.table.max()) < used
    K2, V2, cu2 = cache.read(half.kv_heads, half.d)
    # the others go on, behind what they still share and without sharing
    at = cache.extend([1, 0, 1, 1, 0, 1, 1])
    x5 = rand(5)
    cache_ends = [half(x5, None, at)[0].clone()]
    cache.max_shared = 0
    cache_ends.append(half(x5, None, at)[0].clone())
    assert ((cache_ends[0].double() - cache_ends[1].double()).norm() / cache_ends[1].double().norm()).item() < 2.0 ** -5
    for s in (0, 2, 3, 5, 6):
        assert torch.equal(K2[cu2[s]:cu2[s + 1]], K[cu[s]:cu[s + 1]]) and torch.equal(V2[cu2[s]:cu2[s + 1]], V[cu[s]:cu[s + 1]])


def test_command_runs_with_answers(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["decoder_attention.py", "--sequences", "2", "--context", "200", "--chunk", "64", "--new", "4", "--answers", "3"])
    example.main()
    out = capsys.readouterr().out
    assert "finite True" in out and "3 answers to each of 2 prompts of 200 tokens" in out
