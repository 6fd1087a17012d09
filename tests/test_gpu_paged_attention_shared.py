"""Attention of sequences that share prefixes against the float64 oracle of the paged attention, which knows of no sharing.  The bound is
test_gpu_paged_attention's with its absolute part (a prefix goes the way of chunks); joining parts adds a few float32 roundings, which its 2^-21 holds."""
import numpy as np
import pytest
import torch

import paper_2601_19675_amd as ptq
from test_gpu_paged_attention import LAYOUTS, Problem

pytestmark = pytest.mark.gpu
dev = lambda a: torch.tensor(np.asarray(a, dtype=np.int32), device="cuda")


class Shared(Problem):
    """Sequences of which some lie in groups (first, how many, keys in common); a group's tables name the same pages but for the one in which the
    prefix ends, of which each has a copy."""

    def __init__(self, kv, new, hq, hkv, d, bits, page, groups, **kw):
        super().__init__(kv, new, hq, hkv, d, bits, page, **kw)
        self.groups = groups
        for first, many, common in groups:
            for s in range(first + 1, first + many):
                full, rest = common // page, common % page
                n = min(full, -(-self.kv[s] // page), -(-self.kv[first] // page))
                self.table[s, :n] = self.table[first, :n]
                if rest and n == full and min(self.kv[s], self.kv[first]) > full * page:
                    for c in (self.codes, self.scales, self.zeros):
                        c[:, self.table[s, full], :, :rest] = c[:, self.table[first, full], :, :rest]

    def groups_of(self):
        ends, shared = [self.groups[0][0]], []
        for first, many, common in self.groups:
            if first > ends[-1]:      # sequences between groups are one that shares nothing
                ends.append(first)
                shared.append(0)
            ends.append(first + many)
            shared.append(common)
        return ends, shared

    behind = 1000    # what the bounds leave for keys behind a prefix: below 2048 a workgroup has a sequence's, else all are shared out

    def bounds(self, shared):
        """Few keys of few heads are no work to save: the bounds that the call chooses its way by say that there is more, and sequences that hold nothing and
        ask nothing follow the others.  max_kv, max_shared, how many follow."""
        heads, most = self.codes.shape[2], max(shared, default=0)
        follow = 900 // heads - len(self.kv)
        if most < 64 or follow <= 0:
            return max(self.kv), most, 0
        most = max(most, -(-8_000_000 // (heads * self.d * 2 * self.bits // 8)))    # keys of 8 MB
        return max(max(self.kv), most + self.behind), most, follow

    def run(self, causal=True, window=0, ws=None, ends=None, shared=None, max_shared=None, O=None, loose=True):
        assert window == 0
        if ends is None:
            ends, shared = self.groups_of()
        if loose and max_shared is None:
            max_kv, most, follow = self.bounds(shared)
        else:
            max_kv, most, follow = max(self.kv), max(shared, default=0) if max_shared is None else max_shared, 0
        cu = np.concatenate([self.cu, np.full(follow, self.cu[-1], dtype=self.cu.dtype)])
        table = np.concatenate([self.table, np.zeros((follow, self.table.shape[1]), dtype=self.table.dtype)])
        kv = list(self.kv) + [0] * follow
        q = torch.tensor(self.Q.astype(np.float32), device="cuda").bfloat16()
        O = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda") if O is None else O
        t = lambda a: torch.tensor(a, device="cuda")
        ptq.ptq_paged_attention_shared(q, t(cu), max(self.new), t(self.codes), t(self.scales), t(self.zeros), self.bits, t(table), dev(kv), max_kv, dev(ends),
                                       dev(shared), most, self.scale, O, causal=causal, ws=ws)
        torch.cuda.synchronize()
        return O


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hq,hkv", LAYOUTS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (80, 8), (96, 1), (256, 32), (16, 2), (128, 4), (208, 256)])
def test_layouts(bits, hq, hkv, d, page):
    Shared([333, 301, 500, 200, 150, 90], [1] * 6, hq, hkv, d, bits, page, [(0, 3, 300), (4, 2, 70)], seed=hq * 1000 + d + bits).check(absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("common", [0, 1, 63, 64, 65, 127, 128, 129, 500, 1000, 2047, 2048, 5000, 20000])
def test_prefixes(bits, common):
    Shared([common + 1, common + 40, common + 700], [1, 1, 1], 8, 2, 64, bits, 16, [(0, 3, common)], seed=common).check(absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new", [[2, 1, 4, 3], [4, 4, 0, 1]])
@pytest.mark.parametrize("causal", [True, False])
def test_a_few_tokens(bits, new, causal):
    Shared([1200, 1003, 1500, 30], new, 8, 2, 128, bits, 16, [(0, 3, 1000)], seed=sum(new)).check(causal, absolute=True)


@pytest.mark.parametrize("causal", [True, False])
def test_queries_inside_the_prefix(causal):
    """A sequence that ends before its group's prefix does, one whose new tokens stand in it, one without keys, one with more queries than keys."""
    Shared([400, 200, 258, 0, 2, 256], [2, 2, 4, 1, 4, 3], 4, 1, 64, 8, 16, [(0, 6, 256)], seed=3).check(causal, absolute=True)


@pytest.mark.parametrize("many,hq,hkv,new", [(70, 32, 8, 1), (33, 16, 1, 1), (140, 4, 4, 4), (300, 2, 1, 1)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_more_rows_than_a_tile(many, hq, hkv, new, d):
    kv = [200 + (7 * i) % 90 for i in range(many)]
    Shared(kv, [new] * many, hq, hkv, d, 8, 16, [(0, many, 192)], seed=many).check(absolute=True)


def test_many_groups():
    sizes = [1 + i % 4 for i in range(40)]
    first = np.concatenate(([0], np.cumsum(sizes)))
    kv = [64 * (1 + i % 5) + 3 + i for i in range(int(first[-1]))]
    groups = [(int(first[i]), sizes[i], min(kv[int(first[i]):int(first[i + 1])]) - 2) for i in range(40)]
    Shared(kv, [1] * len(kv), 8, 2, 64, 4, 16, groups, seed=12).check(absolute=True)


def test_a_group_among_sequences_of_none():
    p = Shared([300, 350, 310, 400, 90], [1, 2, 1, 1, 1], 8, 4, 64, 8, 16, [(1, 2, 290)], seed=4)
    p.check(absolute=True)
    plain = Problem.run(p)
    ends, shared = [1, 3], [290]
    got = p.run()
    for s in (0, 3, 4):
        a, b = p.cu[s], p.cu[s + 1]
        assert torch.equal(got[a:b], plain[a:b])
    # groups that are none: before the first sequence, past the last, of one sequence, of a length below 0; no groups at all
    for e, c in (([-1, 3], [290]), ([1, 6], [290]), ([1, 2, 3], [290, 290]), ([1, 3], [-5]), ([1, 1, 1], [290, 290]), ([2], [])):
        assert torch.equal(p.run(ends=e, shared=c, max_shared=290), plain), (e, c)
    assert torch.equal(p.run(ends=[1, 3], shared=[290], max_shared=0), plain)
    # a bound below the prefix: what is past it is each sequence's own
    for bound in (64, 100, 128, 290, 10 ** 8):
        p2 = Shared([300, 350, 310, 400, 90], [1, 2, 1, 1, 1], 8, 4, 64, 8, 16, [(1, 2, 290)], seed=4)
        run = Shared.run
        p2.run = lambda causal=True, window=0, **kw: run(p2, causal, window, ends=ends, shared=shared, max_shared=bound)
        p2.check(absolute=True)


def test_chunks_go_the_usual_way():
    p = Shared([500, 470, 600], [40, 20, 1], 8, 2, 64, 8, 16, [(0, 3, 400)], seed=5)
    assert torch.equal(p.run(loose=False), Problem.run(p))
    p.check(absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kv,groups", [([2600, 2700, 2590, 2650], [(0, 3, 2560)]),            # one of no group among them
                                       ([2650, 2600, 2700, 2590], [(1, 3, 2560)]),
                                       ([3000, 2900, 2800, 2950, 5, 0], [(0, 2, 2752), (2, 2, 64)]),   # behind a long prefix, a short one, none
                                       ([2112, 2048, 2049, 2176, 2177, 4000], [(0, 2, 2048)]),   # behind none: about 2048 keys, and more
                                       ([4300, 4300, 4300], [(0, 2, 4160)])])
@pytest.mark.parametrize("new", [1, 3])
def test_long_sequences_beside_short_ones_behind_a_prefix(bits, kv, groups, new):
    Shared(kv, [min(new, k) for k in kv], 8, 2, 64, bits, 16, groups, seed=len(kv) + new).check(absolute=True)


def test_long_sequences_beside_short_ones_do_not_depend_on_the_workspace():
    p = Shared([2600, 2700, 2590, 2650, 4000], [1, 2, 1, 2, 1], 8, 2, 128, 8, 32, [(0, 3, 2560)], seed=6)
    ws = torch.zeros(ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, 8, 128, sum(p.new), p.bounds(p.groups_of()[1])[0]), dtype=torch.uint8, device="cuda")
    first = p.run(ws=ws)
    for fill in (255, 0x41, 0x7f):
        ws.fill_(fill)
        assert torch.equal(p.run(ws=ws), first)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kv,groups", [([5200, 5300, 5100, 2650], [(0, 3, 2560)]), ([700, 650, 9000, 64, 1], [(0, 2, 600)])])
def test_all_sequences_in_shares(bits, kv, groups):
    p = Shared(kv, [1] * len(kv), 8, 2, 64, bits, 16, groups, seed=len(kv))
    p.behind = 5000
    p.check(absolute=True)


def test_a_workgroup_to_each_and_bounds_below_the_prefix():
    """Bounds of less than 2048 keys; keys from a bound on are each sequence's own."""
    p = Shared([1450, 1500, 1410], [1, 1, 1], 32, 32, 128, 8, 64, [(0, 3, 1400)], seed=3)
    follow = 25
    run = Shared.run

    def bounded(most):
        p.bounds = lambda shared: (1500, most, follow)
        p.run = lambda causal=True, window=0, **kw: run(p, causal, window, **kw)
        p.check(absolute=True)
        return p.run()

    plain = Problem.run(p)
    assert not any(torch.equal(bounded(most), plain) for most in (1400, 1023, 1024))


def test_which_way_it_goes():
    """Outputs of the two ways differ in their roundings: work to save goes through the prefixes apart, little work as in ptq_paged_attention."""
    p = Shared([1300, 1250, 1400, 1211], [1] * 4, 8, 2, 64, 8, 16, [(0, 4, 1200)], seed=2)
    plain = Problem.run(p)
    assert torch.equal(p.run(loose=False), plain)
    assert not torch.equal(p.run(), plain)


@pytest.mark.parametrize("page", [1, 16])
def test_pages_that_are_not_there(page):
    p = Shared([300, 290, 280], [1, 2, 1], 8, 2, 64, 8, page, [(0, 3, 256)], seed=page)
    p.table[:, 100 // page] = -1
    p.table[:, 0] = 2 ** 30
    p.table[1, 270 // page:] = -7
    p.check(absolute=True)
    p = Shared([300, 290, 280], [1, 2, 1], 8, 2, 64, 8, page, [(0, 3, 256)], seed=page)
    p.table = np.ascontiguousarray(p.table[:, :max(1, 130 // page)])     # tables that end inside the prefix
    p.check(absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
def test_what_is_not_seen_has_no_effect(bits):
    p = Shared([330, 200, 259], [1, 2, 3], 4, 2, 64, bits, 16, [(0, 3, 320)], seed=6)
    for j in (261, 300, 319):      # keys of the prefix that only the first sequence sees
        p.scales[:, p.table[0, j // 16], :, j % 16] = np.nan
    p.check(absolute=True)
    clean = Shared([330, 200, 259], [1, 2, 3], 4, 2, 64, bits, 16, [(0, 3, 320)], seed=6).run()
    assert torch.equal(p.run()[1:], clean[1:])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("k_size,v_size", [(40.0, 1.0), (1.0, 1e30), (1.0, 1e-30), (1e-12, 1e5)])
def test_sizes_of_values(bits, k_size, v_size):
    p = Shared([900, 700, 800], [1, 1, 2], 8, 2, 64, bits, 16, [(0, 3, 640)], seed=7, k_size=k_size, v_size=v_size)
    p.check(absolute=True)
    for j in range(640):       # values that grow along the prefix, by far
        p.scales[1, p.table[0, j // 16], :, j % 16] *= np.float32(2.0 ** (j // 40 - 6))
    p.check(absolute=True)


def test_results_do_not_depend_on_the_workspace_or_the_call():
    p = Shared([3000 + 11 * i for i in range(20)], [1] * 20, 8, 2, 128, 8, 16, [(0, 12, 2900), (13, 7, 3000)], seed=8)
    need = ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, 8, 128, 20, p.bounds(p.groups_of()[1])[0])
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    first = p.run(ws=ws)
    assert torch.equal(p.run(ws=ws), first)
    ws.fill_(0x7f)
    assert torch.equal(p.run(ws=ws), first)
    assert torch.equal(p.run(), first)
    with pytest.raises(ptq.PtqError):
        p.run(ws=ws[:need - 256])


def test_replayed_and_on_another_stream():
    p = Shared([700, 650, 690, 720], [1] * 4, 8, 2, 64, 8, 16, [(0, 4, 640)], seed=9)
    t = lambda a: torch.tensor(a, device="cuda")
    Q = torch.tensor(p.Q.astype(np.float32), device="cuda").bfloat16()
    O, want = torch.zeros_like(Q), torch.zeros_like(Q)
    many = 400    # sequences that hold nothing follow, and the bounds are far: work to save
    lens, shared, ends = dev(list(p.kv) + [0] * many), dev([640]), dev([0, 4])
    cache = t(p.codes), t(p.scales), t(p.zeros)
    cu, table = dev(list(p.cu) + [4] * many), t(np.concatenate([p.table, np.zeros((many, p.table.shape[1]), dtype=np.int32)]))
    ws = [torch.empty(ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, 8, 64, 4, 33000), dtype=torch.uint8, device="cuda") for _ in range(2)]
    call = lambda o, w: ptq.ptq_paged_attention_shared(Q, cu, 1, *cache, 8, table, lens, 33000, ends, shared, 32000, p.scale, o, ws=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(O, ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(O, ws[0])
    for i in range(4):
        lens[:4].copy_(dev([c - 5 * i for c in p.kv]))
        shared.fill_(640 - 100 * i)
        graph.replay()
        call(want, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(O, want), i
