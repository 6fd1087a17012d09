"""The attention half of a decoder layer served in 8 bits, with the library's calls one after the other:

    norm and token codes -> query, key and value projections -> keys and values into the paged cache -> attention over the cache
    -> token codes of its output -> output projection

    python examples/decoder_attention.py                     # two prompts in chunks, then single tokens replayed from a graph
    python examples/decoder_attention.py --bits 4 --context 16384 --sequences 16

Weights are random and rounded to the nearest of 255 levels per output channel.  Position encoding is left to the program
around it: it would turn `q` and `k` between the projections and the cache.
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
    """Keys and values of one layer in pages; a sequence takes the next free page when its last one is full."""

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

    def extend(self, new: list[int]) -> dict:
        """Makes room for new[s] more tokens of each sequence; what the calls have to know about these tokens."""
        slots, cu = [], [0]
        for s, n in enumerate(new):
            for j in range(self.lens[s], self.lens[s] + n):
                if j % self.page == 0:
                    self.table[s, j // self.page] = self.free.pop()
                slots.append(int(self.table[s, j // self.page]) * self.page + j % self.page)
            self.lens[s] += n
            cu.append(cu[-1] + n)
        self.table_device.copy_(self.table)   # in place: a graph that was captured goes on reading it
        put = lambda a: torch.tensor(a, dtype=torch.int32, device=self.table_device.device)
        return {"slots": put(slots), "cu_q": put(cu), "max_q": max(new), "kv_lens": put(self.lens)}

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

    def __init__(self, gamma, wqkv, wo, heads: int, kv_heads: int, d: int, cache: PagedCache, max_tokens: int, eps: float = 1e-5):
        self.gamma, self.eps, self.heads, self.kv_heads, self.d, self.cache = gamma, eps, heads, kv_heads, d, cache
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
            need.append(ptq.ptq_workspace_bytes(ptq.OP_PAGED_ATTENTION, heads, d, t, cache.max_kv))
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
        ptq.ptq_kv_cache_write(k, v, at["slots"], c.bits, c.codes, c.scales, c.zeros)
        attended = self.attended[:t]
        ptq.ptq_paged_attention(q, at["cu_q"], at["max_q"], c.codes, c.scales, c.zeros, c.bits, c.table_device, at["kv_lens"], c.max_kv,
                                d ** -0.5, attended, ws=self.ws)
        codes = self.attended_codes[:t]
        ptq.ptq_rmsnorm_quantize(attended.view(t, h * d), codes, scales, normalize=False)
        ptq.ptq_int8_linear(codes, scales, self.wo, self.wo_scales, self.out[:t], ws=self.ws)
        return self.out[:t], total


def make_half(hidden=4096, heads=32, kv_heads=8, d=128, bits=8, page=32, sequences=2, max_kv=4096, max_tokens=2048, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    wqkv = rand((heads + 2 * kv_heads) * d, hidden) * hidden ** -0.5
    wo = rand(hidden, heads * d) * (heads * d) ** -0.5
    gamma = (1.0 + 0.1 * rand(hidden)).bfloat16()
    cache = PagedCache(sequences, max_kv, kv_heads, d, bits, page)
    return AttentionHalf(gamma, wqkv, wo, heads, kv_heads, d, cache, max_tokens), (gamma, wqkv, wo)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--sequences", type=int, default=2)
    p.add_argument("--context", type=int, default=4096, help="tokens of a prompt; a few fewer than the cache holds")
    p.add_argument("--chunk", type=int, default=1024, help="tokens of a prompt that go through at a time")
    p.add_argument("--bits", type=int, default=8, choices=(4, 8))
    p.add_argument("--new", type=int, default=32, help="single tokens afterwards")
    a = p.parse_args()
    half, _ = make_half(bits=a.bits, sequences=a.sequences, max_kv=a.context + a.new + 1, max_tokens=a.sequences * a.chunk)
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


if __name__ == "__main__":
    main()
