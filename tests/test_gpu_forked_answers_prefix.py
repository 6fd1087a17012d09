"""Forks, released and taken slots, compaction and a captured step with the attention going through shared prefixes apart.  What the calls choose their way
by says that there is work to save: sequences that hold nothing follow, and the bounds are far.  Bounds: as in test_gpu_forked_answers_example.py."""
import pytest
import torch

import paper_2601_19675_amd as ptq
from test_gpu_decoder_attention_example import BOUND, example
from test_gpu_forked_answers_example import plain

pytestmark = pytest.mark.gpu
SEQUENCES, FAR_SHARED, FAR_KV = 64, 40000, 41000


def make(bits):
    half, (gamma, _, _) = example.make_half(hidden=512, heads=8, kv_heads=2, d=64, page=16, max_kv=500, max_tokens=700, rotary=True, whole_prompts=True, bits=bits,
                                            seed=bits, sequences=SEQUENCES)
    half.ws = torch.empty(ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, 8, 64, SEQUENCES, FAR_KV), dtype=torch.uint8, device="cuda")
    half.cache.max_kv = FAR_KV
    g = torch.Generator(device="cuda").manual_seed(5)
    return half, gamma, lambda n: torch.randn(n, 512, device="cuda", generator=g).bfloat16()


def counts(of):
    return [of.get(s, 0) for s in range(SEQUENCES)]


def apart_from_each_other(half, x, at, mine):
    """The same tokens with every context gone through by itself: close, and not the same bits, or nothing was shared."""
    shared, half.cache.max_shared = half.cache.max_shared, 0
    other = half(x, None, at)[0].clone()
    half.cache.max_shared = shared
    assert not torch.equal(mine, other)
    assert ((mine.double() - other.double()).norm() / other.double().norm()).item() < 2.0 ** -5


def near(half, gamma, got, tokens, bits):
    want = plain(half, gamma, torch.cat(tokens), None)[-len(got):]
    o = torch.cat(got).double().cpu()
    assert ((o - want).norm() / want.norm()).item() < BOUND[bits]


@pytest.mark.parametrize("bits", [8, 4])
def test_answers(bits):
    half, gamma, rand = make(bits)
    cache, parent = half.cache, [0, 0, 0, 3, 4, 4, 4]
    prompts = {0: rand(300), 3: rand(37), 4: rand(210)}
    half(torch.cat([prompts[s] for s in (0, 3, 4)]), None, cache.extend(counts({0: 300, 3: 37, 4: 210})))
    cache.fork([[0, 1, 2], [4, 5, 6]])
    cache.max_shared = FAR_SHARED
    one = counts({s: 1 for s in range(7)})
    tokens, got, x, graph = [[prompts[parent[s]]] for s in range(7)], [[] for _ in range(7)], rand(7), None
    at = cache.extend(one)
    for step in range(6):
        if step:
            x.copy_(rand(7))
            now = cache.extend(one)
            for name in ("slots", "kv_lens", "positions"):
                at[name].copy_(now[name])
        if step == 2:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                half(x, None, at)
        if graph is None:
            half(x, None, at)
        else:
            graph.replay()
        for s in range(7):
            tokens[s].append(x[s:s + 1].clone())
            got[s].append(half.out[s:s + 1].clone())
    replayed = half.out[:7].clone()
    assert torch.equal(half(x, None, at)[0], replayed)
    for s in range(7):
        near(half, gamma, got[s], tokens[s], bits)
    apart_from_each_other(half, x, at, replayed)
    # a family's parent goes and a fork, pages move together
    cache.release(4)
    cache.release(1)
    cache.compact()
    left = [0, 2, 3, 5, 6]
    x5 = rand(5)
    at = cache.extend(counts({s: 1 for s in left}))
    out = half(x5, None, at)[0].clone()
    for i, s in enumerate(left):
        near(half, gamma, [out[i:i + 1]], tokens[s] + [x5[i:i + 1]], bits)
    apart_from_each_other(half, x5, at, out)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("gone", [0, 2, 4])
def test_a_slot_taken_by_another_sequence(bits, gone):
    """A fork, or the parent, goes, and another prompt comes into its slot, between sequences that still lie behind what they share."""
    half, gamma, rand = make(bits)
    cache, tokens = half.cache, [[rand(300)] for _ in range(5)]
    half(tokens[0][0], None, cache.extend(counts({0: 300})))
    cache.fork([[0, 1, 2, 3, 4]])
    cache.max_shared = FAR_SHARED
    for s in range(1, 5):
        tokens[s] = [tokens[0][0]]

    def step():
        x = rand(5)
        at = cache.extend(counts({s: 1 for s in range(5)}))
        out = half(x, None, at)[0].clone()
        for s in range(5):
            tokens[s].append(x[s:s + 1])
            near(half, gamma, [out[s:s + 1]], tokens[s], bits)
        apart_from_each_other(half, x, at, out)
    step()
    cache.release(gone)
    tokens[gone] = [rand(350)]
    half(tokens[gone][0], None, cache.extend(counts({gone: 350})))
    step()
    step()
