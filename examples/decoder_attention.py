"""The attention half of a decoder layer served in 8 bits, with the library's calls one after the other:

    norm and token codes -> query, key and value projections -> rotary positions, keys and values into the paged cache
    -> attention over the cache -> token codes of its output -> output projection

    python examples/decoder_attention.py                     # two prompts in chunks, then single tokens replayed from a graph
    python examples/decoder_attention.py --bits 4 --context 16384 --sequences 16
    python examples/decoder_attention.py --answers 16        # and then every prompt forked, its answers decoded behind what they share

Weights are random and rounded to the nearest of 255 levels per output channel.  A half without frequencies leaves the position encoding
to the program around it.  With whole_prompts, prompts that come in one piece attend to their keys and values before those are quantized.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2601_19675_amd as ptq  # noqa: E402


def quantize_weight(W: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """int8 codes and float32 scales, one per output channel, of W (out x in)."""
    scales = W.float().abs().amax(dim=1).clamp_min(1e-30) / 127.0
    return (W.float() / scales[:, None]).round().clamp(-127, 127).to(torch.int8), scales


class PagedCache:
    """Keys and values of one layer in pages; a sequence takes the next free page when its last one is full, forks of it share its full pages."""

    def __init__(self, sequences: int, max_kv: int, heads: int, d: int, bits: int, page: int, device="cuda"):
        per = -(-max_kv // page)
        pages = sequences * per
        self.bits, self.page, self.max_kv = bits, page, max_kv
        self.codes = torch.zeros(2, pages, heads, page, d * bits // 8, dtype=torch.uint8, device=device)
        self.scales = torch.zeros(2, pages, heads, page, device=device)
        self.zeros = torch.zeros(2, pages, heads, page, dtype=torch.uint8, device=device)
        self.table = torch.full((sequences, per), -1, dtype=torch.int32)
        self.table_device = self.table.to(device)
        self.lens = [0] * sequences
        self.free = list(range(pages))[::-1]
        self.users = [0] * pages
        self.behind = [False] * sequences   # whether it still is the fork, or the parent, that its family began with
        self.families, self.groups_device, self.shared_device, self.max_shared = [], None, None, 0
        self.outdated = []   # what graphs of before a fork may still read: that nothing is shared

    def _put(self, a) -> torch.Tensor:
        return torch.tensor(a, dtype=torch.int32, device=self.table_device.device)

    def _take(self) -> int:
        page = self.free.pop()
        self.users[page] = 1
        return page

    def extend(self, new: list[int]) -> dict:
        """Makes room for new[s] more tokens of each sequence; what the calls have to know about these tokens."""
        slots, cu, positions, whole = [], [0], [], all(n == 0 or self.lens[s] == 0 for s, n in enumerate(new))
        taken = any(n > 0 and self.lens[s] == 0 for s, n in enumerate(new))
        for s, n in enumerate(new):
            for j in range(self.lens[s], self.lens[s] + n):
                if j % self.page == 0:
                    self.table[s, j // self.page] = self._take()
                slots.append(int(self.table[s, j // self.page]) * self.page + j % self.page)
                positions.append(j)
            self.lens[s] += n
            cu.append(cu[-1] + n)
        self.table_device.copy_(self.table)   # in place: a graph that was captured goes on reading it
        if taken:
            self._share()
        return {"slots": self._put(slots), "cu_q": self._put(cu), "max_q": max(new), "kv_lens": self._put(self.lens),
                "positions": self._put(positions), "whole": whole}

    def release(self, s: int) -> None:
        """Sequence s is gone; pages that nobody else has are free again, and s is there for another sequence."""
        for i in range(-(-self.lens[s] // self.page)):
            page = int(self.table[s, i])
            self.users[page] -= 1
            if self.users[page] == 0:
                self.free.append(page)
        self.table[s] = -1
        self.lens[s] = 0
        self.behind[s] = False
        self.table_device.copy_(self.table)
        self._share()

    def _share(self) -> None:
        """Tells the attention which sequences lie behind what: between families there are groups that share nothing.  Of a family it is the longest run of
        members that no other sequence has come between (one that holds nothing may lie there).  It begins with a member, whose pages are the
        ones that are read."""
        if not self.families:
            return
        cu, shared = [0], []
        for family, length in self.families:
            runs = [[]]
            for s in family:
                if self.behind[s]:
                    runs[-1].append(s)
                elif self.lens[s] > 0:
                    runs.append([])
            run = max(runs, key=len)
            cu += [run[0], run[-1] + 1] if run else [family[0], family[0]]
            shared += [0, length if run else 0]
        if self.shared_device is not None and len(shared) == len(self.shared_device):   # in place, as the table
            self.groups_device.copy_(self._put(cu))
            self.shared_device.copy_(self._put(shared))
            return
        if self.shared_device is not None:
            self.shared_device.zero_()
            self.outdated.append((self.groups_device, self.shared_device))
        self.groups_device, self.shared_device = self._put(cu), self._put(shared)

    def fork(self, families: list[list[int]]) -> None:
        """families[j] = [sequence, forks ...]: the forks, empty ones that follow it, become copies of the sequence.  Full pages are shared, the page in which
        it goes on is copied.  From now on the attention goes through what a family has in common once for all of it."""
        source, target = [], []
        for family in families:
            parent, length = family[0], self.lens[family[0]]
            assert family == list(range(parent, parent + len(family)))
            for s in family[1:]:
                assert self.lens[s] == 0
                for i in range(-(-length // self.page)):
                    page = int(self.table[parent, i])
                    if (i + 1) * self.page <= length:
                        self.users[page] += 1
                    else:
                        source.append(page)
                        page = self._take()
                        target.append(page)
                    self.table[s, i] = page
                self.lens[s] = length
        if source:
            cache = self.codes, self.scales, self.zeros
            ptq.ptq_kv_cache_copy_pages(*cache, self._put(source), *cache, self._put(target))
        self.table_device.copy_(self.table)
        self.families = [(family, self.lens[family[0]]) for family in families]
        self.behind = [any(s in family and length > 0 for family, length in self.families) for s in range(len(self.lens))]
        self.max_shared = max(length for _, length in self.families)
        self._share()

    def compact(self) -> None:
        """Brings the pages that are in use together at the beginning."""
        used = [p for p, n in enumerate(self.users) if n]
        gaps = [p for p in range(len(used)) if not self.users[p]]
        moved = dict(zip([p for p in used if p >= len(used)], gaps))
        if not moved:
            return
        cache = self.codes, self.scales, self.zeros
        ptq.ptq_kv_cache_copy_pages(*cache, self._put(list(moved)), *cache, self._put(list(moved.values())))
        for old, now in moved.items():
            self.users[now], self.users[old] = self.users[old], 0
        self.free = [p for p in range(len(self.users))[::-1] if not self.users[p]]
        self.table.apply_(lambda p: moved.get(p, p))
        self.table_device.copy_(self.table)

    def read(self, heads: int, d: int) -> tuple[torch.Tensor, torch.Tensor, list[int]]:
        """All sequences' keys and values, one after the other, and where each begins."""
        cu = [0]
        for n in self.lens:
            cu.append(cu[-1] + n)
        K = torch.empty(cu[-1], heads, d, dtype=torch.bfloat16, device=self.codes.device)
        V = torch.empty_like(K)
        ptq.ptq_kv_cache_read(self.codes, self.scales, self.zeros, self.bits, self.table_device,
                              torch.tensor(cu, dtype=torch.int32, device=K.device), max(self.lens), K, V)
        return K, V, cu


class AttentionHalf:
    """hidden -> heads of d channels over kv_heads -> hidden; every call's outputs go where they went the last time."""

    def __init__(self, gamma, wqkv, wo, heads: int, kv_heads: int, d: int, cache: PagedCache, max_tokens: int, eps: float = 1e-5,
                 freq: torch.Tensor | None = None, magnitude: float = 1.0, whole_prompts: bool = False):
        self.gamma, self.eps, self.heads, self.kv_heads, self.d, self.cache = gamma, eps, heads, kv_heads, d, cache
        self.freq, self.magnitude, self.whole_prompts = freq, magnitude, whole_prompts
        self.wqkv, self.wqkv_scales = quantize_weight(wqkv)
        self.wo, self.wo_scales = quantize_weight(wo)
        hidden, dev = wqkv.shape[1], wqkv.device
        bf16 = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device=dev)
        self.codes = torch.empty(max_tokens, hidden, dtype=torch.int8, device=dev)
        self.attended_codes = torch.empty(max_tokens, heads * d, dtype=torch.int8, device=dev)
        self.scales = torch.empty(max_tokens, device=dev)
        self.residual, self.qkv = bf16(max_tokens, hidden), bf16(max_tokens, (heads + 2 * kv_heads) * d)
        self.attended, self.out = bf16(max_tokens, heads, d), bf16(max_tokens, hidden)
        need = []   # (the most is not always at the most tokens)
        for t in range(1, max_tokens + 1):
            need += [ptq.ptq_workspace_bytes(ptq.OP_INT8_LINEAR, *w.shape, t) for w in (self.wqkv, self.wo)]
            need += [ptq.ptq_workspace_bytes(op, heads, d, t, cache.max_kv) for op in (ptq.OP_PAGED_ATTENTION, ptq.OP_SHARED_ATTENTION)]
        self.ws = torch.empty(max(256, *need), dtype=torch.uint8, device=dev)

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None, at: dict) -> tuple[torch.Tensor, torch.Tensor]:
        """x (tokens x hidden, bfloat16), the sum of the layers before or None, what PagedCache.extend said of the tokens;
        returns the half's output and the sum x + residual that it is to be added to."""
        t, c, h, g, d = x.shape[0], self.cache, self.heads, self.kv_heads, self.d
        codes, scales, qkv = self.codes[:t], self.scales[:t], self.qkv[:t]
        total = x if residual is None else self.residual[:t]
        ptq.ptq_rmsnorm_quantize(x, codes, scales, gamma=self.gamma, residual=residual, residual_out=None if residual is None else total,
                                 eps=self.eps)
        ptq.ptq_int8_linear(codes, scales, self.wqkv, self.wqkv_scales, qkv, ws=self.ws)
        q, k, v = (p.view(t, -1, d) for p in qkv.split([h * d, g * d, g * d], dim=1))   # strided views: nothing is copied
        attended, scale, whole = self.attended[:t], d ** -0.5, self.whole_prompts and at["whole"]
        if self.freq is None or whole:
            if self.freq is not None:
                turned = qkv[:, :(h + g) * d].view(t, h + g, d)   # queries and keys, where they lie
                ptq.ptq_rotary(turned, at["positions"], self.freq, turned, scale=self.magnitude)
            ptq.ptq_kv_cache_write(k, v, at["slots"], c.bits, c.codes, c.scales, c.zeros)
        else:
            ptq.ptq_rotary_kv_cache_write(q, k, v, at["positions"], self.freq, at["slots"], c.bits, c.codes, c.scales, c.zeros, q, scale=self.magnitude)
        if whole:
            ptq.ptq_prompt_attention(q, k, v, at["cu_q"], at["max_q"], scale, attended)
        elif c.max_shared > 0:
            ptq.ptq_paged_attention_shared(q, at["cu_q"], at["max_q"], c.codes, c.scales, c.zeros, c.bits, c.table_device, at["kv_lens"], c.max_kv,
                                           c.groups_device, c.shared_device, c.max_shared, scale, attended, ws=self.ws)
        else:
            ptq.ptq_paged_attention(q, at["cu_q"], at["max_q"], c.codes, c.scales, c.zeros, c.bits, c.table_device, at["kv_lens"], c.max_kv,
                                    scale, attended, ws=self.ws)
        codes = self.attended_codes[:t]
        ptq.ptq_rmsnorm_quantize(attended.view(t, h * d), codes, scales, normalize=False)
        ptq.ptq_int8_linear(codes, scales, self.wo, self.wo_scales, self.out[:t], ws=self.ws)
        return self.out[:t], total


def make_half(hidden=4096, heads=32, kv_heads=8, d=128, bits=8, page=32, sequences=2, max_kv=4096, max_tokens=2048, seed=0, rotary=False,
              whole_prompts=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    wqkv = rand((heads + 2 * kv_heads) * d, hidden) * hidden ** -0.5
    wo = rand(hidden, heads * d) * (heads * d) ** -0.5
    gamma = (1.0 + 0.1 * rand(hidden)).bfloat16()
    cache = PagedCache(sequences, max_kv, kv_heads, d, bits, page)
    freq = ptq.ptq_rotary_frequencies(d).to("cuda") if rotary else None
    return AttentionHalf(gamma, wqkv, wo, heads, kv_heads, d, cache, max_tokens, freq=freq, whole_prompts=whole_prompts), (gamma, wqkv, wo)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--sequences", type=int, default=2)
    p.add_argument("--context", type=int, default=4096, help="tokens of a prompt; a few fewer than the cache holds")
    p.add_argument("--chunk", type=int, default=1024, help="tokens of a prompt that go through at a time")
    p.add_argument("--bits", type=int, default=8, choices=(4, 8))
    p.add_argument("--new", type=int, default=32, help="single tokens afterwards")
    p.add_argument("--answers", type=int, default=0, help="forks of every prompt, decoded afterwards")
    a = p.parse_args()
    half, _ = make_half(bits=a.bits, sequences=a.sequences, max_kv=a.context + a.new + 1, max_tokens=a.sequences * a.chunk, rotary=True,
                        whole_prompts=True)
    cache, dev = half.cache, "cuda"
    clock = lambda: torch.cuda.Event(enable_timing=True)

    begin, end, done = clock(), clock(), 0
    x = torch.randn(a.sequences * a.chunk, 4096, device=dev).bfloat16()
    chunks = []   # what the host has to say is laid out first
    while done < a.context:
        n = min(a.chunk, a.context - done)
        chunks.append((n * a.sequences, cache.extend([n] * a.sequences)))
        done += n
    begin.record()
    for t, at in chunks:
        half(x[:t], None, at)
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end)
    print(f"{a.sequences} prompts of {a.context} tokens in chunks of {a.chunk}: {ms:.2f} ms, {a.sequences * a.context / ms * 1e3:.0f} tokens/s of a layer's half")

    # single tokens: one graph, whose inputs are written where it reads them
    x1, r1 = torch.randn(a.sequences, 4096, device=dev).bfloat16(), torch.randn(a.sequences, 4096, device=dev).bfloat16()
    at = cache.extend([1] * a.sequences)
    half(x1, r1, at)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        half(x1, r1, at)
    begin.record()
    for _ in range(a.new):
        now = cache.extend([1] * a.sequences)
        at["slots"].copy_(now["slots"])
        at["kv_lens"].copy_(now["kv_lens"])
        at["positions"].copy_(now["positions"])
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    whole = begin.elapsed_time(end) / a.new * 1e3
    begin.record()
    for _ in range(100):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print(f"single tokens at {cache.lens[0]} tokens of context: {begin.elapsed_time(end) * 10:.1f} us a step on the device, "
          f"{whole:.1f} us with the host's bookkeeping")
    K, V, cu = cache.read(half.kv_heads, half.d)
    kv_bytes = cache.codes.numel() + 4 * cache.scales.numel() + cache.zeros.numel()
    print(f"cache: {kv_bytes / 1e6:.1f} MB for what bfloat16 holds in {2 * 2 * K.numel() / 1e6:.1f} MB; "
          f"read back: keys {tuple(K.shape)}, finite {bool(torch.isfinite(K).all() & torch.isfinite(V).all())}")
    if a.answers:
        answers(a)


def answers(a):
    """Prompts in one piece each, forked, and a token of every answer decoded with what a family has in common gone through once, and without."""
    n = a.sequences * a.answers
    half, _ = make_half(bits=a.bits, sequences=n, max_kv=a.context + a.new + 1, max_tokens=max(n, a.context), rotary=True, whole_prompts=True)
    cache, families = half.cache, [list(range(s, s + a.answers)) for s in range(0, n, a.answers)]
    for family in families:
        new = [0] * n
        new[family[0]] = a.context
        half(torch.randn(a.context, 4096, device="cuda").bfloat16(), None, cache.extend(new))
    cache.fork(families)
    x = torch.randn(n, 4096, device="cuda").bfloat16()
    for _ in range(a.new - 1):
        half(x, x, cache.extend([1] * n))
    at = cache.extend([1] * n)
    shared, took = cache.max_shared, {}
    for way in ("apart", "shared"):
        cache.max_shared = shared if way == "shared" else 0
        half(x, x, at)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            half(x, x, at)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(100):
            graph.replay()
        end.record()
        torch.cuda.synchronize()
        took[way] = begin.elapsed_time(end) * 10
    pages = sum(1 for u in cache.users if u)
    print(f"{a.answers} answers to each of {a.sequences} prompts of {a.context} tokens: {took['shared']:.1f} us a step, {took['apart']:.1f} us with every "
          f"context by itself; {pages} pages in place of {n * -(-cache.lens[0] // cache.page)}")


if __name__ == "__main__":
    main()
