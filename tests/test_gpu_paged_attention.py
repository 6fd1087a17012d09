"""Attention over the paged quantized cache against its float64 oracle: single tokens, chunks, every head layout, windows, pages
that end inside tiles or are not there, rows that see nothing, NaN in what is not seen."""
import numpy as np
import pytest
import torch

import paper_2601_19675_amd as ptq
from oracle import attention_oracle as orc

pytestmark = pytest.mark.gpu


class Problem:
    """A filled cache and queries; lengths and new tokens per sequence."""

    def __init__(self, kv, new, hq, hkv, d, bits, page, seed=0, k_size=1.0, v_size=1.0, q_size=1.0, extra=2):
        g = np.random.default_rng(seed)
        self.kv, self.new, self.hq, self.d, self.bits = list(kv), list(new), hq, d, bits
        per = max(1, max(-(-c // page) for c in kv))
        used = [-(-c // page) for c in kv]
        pages = sum(used) + extra
        order = g.permutation(pages).astype(np.int32)
        self.table = np.full((len(kv), per), 2 ** 31 - 1, dtype=np.int32)
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = order[at:at + u]
            at += u
        shape = (2, pages, hkv, page)
        x = g.standard_normal(shape + (d,)) * np.exp(0.4 * g.standard_normal(d))
        x = x * np.array([k_size, v_size]).reshape(2, 1, 1, 1, 1)
        top = 2 ** bits - 1
        lo, hi = np.minimum(x.min(-1), 0), np.maximum(x.max(-1), 0)
        self.scales = ((hi - lo) / top).astype(np.float32)
        self.zeros = np.rint(-lo / self.scales).astype(np.uint8)
        c = np.clip(np.rint(x / self.scales[..., None]) + self.zeros[..., None], 0, top).astype(np.int64)
        if bits == 8:
            self.codes = c.astype(np.uint8)
        else:
            i = np.arange(8)
            w = (c.reshape(shape + (d // 8, 8)) << (4 * (i // 2) + 16 * (i % 2))).sum(-1)
            self.codes = w.astype("<u4").view(np.uint8).reshape(shape + (d // 2,))
        self.cu = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        self.Q = orc.store(q_size * g.standard_normal((int(self.cu[-1]), hq, d)), "bf16")
        self.scale = 1.0 / np.sqrt(d)

    def run(self, causal=True, window=0, strided=False, ws=None, O=None):
        dev = lambda a, **kw: torch.tensor(a, device="cuda", **kw)
        t = self.Q.shape[0]
        if strided:   # queries inside a fused projection's rows, heads further apart than d
            base = torch.zeros((t, self.hq + 2, self.d + 8), dtype=torch.bfloat16, device="cuda")
            base[:, 1:-1, 4:-4] = dev(self.Q.astype(np.float32)).bfloat16()
            Q, O = base[:, 1:-1, 4:-4], torch.full((t, self.hq, self.d + 4), 5.0, dtype=torch.bfloat16, device="cuda")[:, :, :self.d]
        else:
            Q = dev(self.Q.astype(np.float32)).bfloat16()
            O = torch.full((t, self.hq, self.d), 5.0, dtype=torch.bfloat16, device="cuda") if O is None else O
        ptq.ptq_paged_attention(Q, dev(self.cu), max(self.new), dev(self.codes), dev(self.scales), dev(self.zeros), self.bits,
                                dev(self.table), dev(np.array(self.kv, dtype=np.int32)), max(self.kv), self.scale, O, causal=causal,
                                window=window, ws=ws)
        torch.cuda.synchronize()
        return O

    def check(self, causal=True, window=0, absolute=False, **kw):
        got = self.run(causal, window, **kw).double().cpu().numpy()
        want, size, reach = orc.attention(self.Q, self.cu, self.codes, self.scales, self.zeros, self.bits, self.table, self.kv,
                                          self.scale, causal, window, spread=True)
        # bfloat16 rounds once (2^-8).  Weights: float16 (2^-11 of a weight; values in float16 twice more, scale and product; the
        # smallest weights absolutely, 2^-24 each), and the score's float32 sums, in numerator and denominator.
        rel = 3 * 2.0 ** -11 + max(self.kv) * 2.0 ** -24 + 2 * ((self.d + 8) * 2.0 ** -24 * reach[..., None] + 2.0 ** -21)
        tol = 2.0 ** -8 * np.abs(want) * 1.01 + rel * size + 1e-37
        if absolute:   # half of float16's smallest number of the largest weight, for every key, of the largest value
            top = np.abs(self.scales[1].astype(np.float64)) * np.maximum(self.zeros[1], 2 ** self.bits - 1 - self.zeros[1].astype(np.int64))
            tol += max(self.kv) * 2.0 ** -24 * np.nanmax(np.where(np.isinf(top), np.nan, top))
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(got), nan)
        bad = ~nan & ~(np.abs(got - want) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])


# One key takes all the weight here, and where its value is 0 (often, of 4 bits) the others' weights of less than 2^-24 would have to show: they are
# rounded to float16, absolutely.  The bound of `check` counts that relative to sum p |v| and is missed; test_scores_far_apart has
# the same inputs against an absolute one.
VANISH = pytest.mark.xfail(strict=False, reason="weights below float16's smallest number vanish")
LAYOUTS = [(4, 4), (8, 2), (28, 4), (16, 1), (3, 3)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hq,hkv", LAYOUTS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (80, 8), (96, 1), (256, 32), (16, 2), (128, 4), (208, 256)])
def test_single_tokens(bits, hq, hkv, d, page):
    Problem([1, 37, 700, 64, 257], [1] * 5, hq, hkv, d, bits, page, seed=hq * 1000 + d + bits).check(strided=page == 8)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kv", [1, 2, 31, 32, 33, 127, 128, 129, 255, 256, 257, 3000, 20000])
def test_lengths(bits, kv):
    Problem([kv, max(1, kv // 3)], [1, 1], 8, 2, 64, bits, 16, seed=kv).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new", [[2, 1, 4], [4, 4, 0]])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5), (True, 300), (False, 7), (True, 1)])
def test_a_few_tokens(bits, new, causal, window):
    Problem([200, 3, 1500], new, 8, 2, 128, bits, 16, seed=window).check(causal, window)


def test_more_queries_than_keys_see_nothing():
    # the first queries stand before the first key; a sequence without keys
    Problem([2, 0, 40], [4, 3, 1], 4, 4, 64, 8, 16).check()
    Problem([0, 0], [1, 1], 4, 4, 64, 8, 16).check()


@pytest.mark.parametrize("page", [1, 16, 64])
def test_pages_that_are_not_there(page):
    p = Problem([300, 190, 70], [1, 2, 1], 8, 2, 64, 8, page, seed=page)
    per = p.table.shape[1]
    p.table[0, per // 2], p.table[1, 0], p.table[2, :] = -1, 2 ** 30, -7
    p.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page", [1, 16])
def test_what_is_not_seen_has_no_effect(bits, page):
    p = Problem([61, 130, 47], [2, 1, 4], 4, 2, 64, bits, page, seed=3)
    g = np.random.default_rng(1)
    held = np.zeros(p.scales.shape, dtype=bool)   # rows of some sequence
    for s, c in enumerate(p.kv):
        for j in range(c):
            held[:, p.table[s, j // page], :, j % page] = True
    p.scales[~held] = np.where(g.random((~held).sum()) < 0.5, np.nan, np.inf)
    p.codes[~held] = 255
    p.check()
    # a token whose key or value was not finite: queries that see it become NaN, those before it do not
    p.scales[0, p.table[2, 45 // page], 0, 45 % page] = np.nan
    p.scales[1, p.table[0, 60 // page], 1, 60 % page] = np.nan
    p.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("k_size,v_size,q_size", [(1.0, 1e6, 1.0), (1.0, 1e-9, 1.0), pytest.param(40.0, 1.0, 10.0, marks=VANISH), (1e-12, 1.0, 1e12), (1e10, 1.0, 1e-10),
                                                  (0.0, 1.0, 1.0), (1.0, 1e30, 1.0), (1.0, 1e-33, 1.0)])
def test_sizes_of_values(bits, k_size, v_size, q_size):
    p = Problem([513, 60], [1, 2], 8, 4, 64, bits, 16, seed=5, k_size=max(k_size, 1e-30), v_size=v_size, q_size=q_size)
    # values of very different sizes from key to key
    p.scales[1] *= np.exp2(np.random.default_rng(2).integers(-12, 12, p.scales[1].shape)).astype(np.float32)
    p.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_scores_far_apart(bits):
    p = Problem([513, 60], [1, 2], 8, 4, 64, bits, 16, seed=5, k_size=40.0, q_size=10.0)
    p.scales[1] *= np.exp2(np.random.default_rng(2).integers(-12, 12, p.scales[1].shape)).astype(np.float32)
    p.check(absolute=True)


def test_queries_of_different_sizes_share_a_tile():
    p = Problem([400, 90], [2, 1], 8, 2, 128, 8, 16, seed=6)
    p.Q = orc.store(p.Q * np.exp2(np.random.default_rng(3).integers(-60, 5, p.Q.shape[:2]))[..., None], "bf16")
    p.Q[0, 3] = 0.0
    p.check()


@pytest.mark.parametrize("new", [[1, 1], [2, 1]])
def test_its_stream_and_graph(new):
    p = Problem([4000, 900], new, 8, 2, 128, 8, 16, seed=7)
    want = p.run().clone()
    need = max(256, ptq.ptq_workspace_bytes(ptq.OP_PAGED_ATTENTION, 8, 128, p.Q.shape[0], 4000))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN, if it were read
    assert torch.equal(p.run(ws=ws), want)
    dev = lambda a: torch.tensor(a, device="cuda")
    Q = dev(p.Q.astype(np.float32)).bfloat16()
    args = (Q, dev(p.cu), max(new), dev(p.codes), dev(p.scales), dev(p.zeros), 8, dev(p.table), dev(np.array(p.kv, dtype=np.int32)),
            4000, p.scale)
    O = torch.zeros_like(Q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ptq.ptq_paged_attention(*args, O, ws=ws)
    s.synchronize()
    assert torch.equal(O, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ptq.ptq_paged_attention(*args, O, ws=ws)
    for _ in range(3):
        O.zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)


def test_sequences_that_do_not_fit_are_left_out():
    p = Problem([50, 50, 50], [1, 1, 1], 4, 4, 64, 8, 16, seed=8)
    ok = p.run().clone()
    p.cu[3] = 9   # past the tokens there are
    O = p.run(O=torch.full_like(ok, 5.0))
    assert torch.equal(O[:2], ok[:2]) and (O[2] == 5.0).all()


@pytest.mark.parametrize("hq,hkv,d,bits,page,window", [(4, 2, 64, 4, 16, 0), (8, 8, 128, 8, 64, 0), (16, 1, 64, 8, 1, 0), (8, 2, 64, 8, 16, 2100)])
def test_contexts_of_many_sequences_are_dealt_out(hq, hkv, d, bits, page, window):
    # more sequences than a wave looks at together, some without queries or keys, shares that end anywhere
    g = np.random.default_rng(hq + d)
    kv = [int(c) for c in np.exp(g.uniform(0, np.log(5000), 69))] + [0, 6000, 1, 0]
    new = [1] * len(kv)
    new[5] = new[40] = new[71] = 0
    Problem(kv, new, hq, hkv, d, bits, page, seed=hq).check(True, window, absolute=True)
