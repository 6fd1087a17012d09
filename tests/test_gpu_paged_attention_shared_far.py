"""Prefixes whose work is more than 32 bits count: the call is ptq_paged_attention, and the workspace's old contents do not reach the outputs."""
import pytest
import torch

import paper_2601_19675_amd as ptq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fill", [0x7f, 0xff, 0])
def test_more_work_than_32_bits_count(fill):
    """128 pairs of sequences, 2048 heads, 2^19 keys to a prefix: 128 tiles of rows x 2048 x 2^13 tiles of keys are 2^31.  The sequences themselves hold
    few keys, all of them in one page; 768 that hold nothing follow, so that the bounds say that prefixes apart would save time."""
    heads, d, page, pairs, keys, follow = 2048, 16, 256, 128, 2 ** 19, 768
    g = torch.Generator(device="cuda").manual_seed(7)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    codes = torch.randint(0, 256, (2, 1, heads, page, d), dtype=torch.uint8, device="cuda", generator=g)
    scales = 0.01 + 0.01 * torch.rand(2, 1, heads, page, device="cuda", generator=g)
    zeros = torch.randint(100, 150, (2, 1, heads, page), dtype=torch.uint8, device="cuda", generator=g)
    t, b = 2 * pairs, 2 * pairs + follow
    Q = torch.randn(t, heads, d, device="cuda", generator=g).bfloat16()
    table = torch.zeros(b, keys // page, dtype=torch.int32, device="cuda")
    cu, lens = ints(list(range(t + 1)) + [t] * follow), ints([65 + i % 100 for i in range(t)] + [0] * follow)
    ends, shared = ints(list(range(0, t + 1, 2))), ints([keys] * pairs)
    cache = (Q, cu, 1, codes, scales, zeros, 8, table, lens, keys)
    want, got = torch.zeros_like(Q), torch.full_like(Q, 3.0)
    ptq.ptq_paged_attention(*cache, d ** -0.5, want)
    ws = torch.full((ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, heads, d, t, keys),), fill, dtype=torch.uint8, device="cuda")
    ptq.ptq_paged_attention_shared(*cache, ends, shared, keys, d ** -0.5, got, ws=ws)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(want).all()) and bool((want != 0).any())
    assert torch.equal(got, want)
