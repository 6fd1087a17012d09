"""Chunks of tokens over the paged quantized cache against the float64 oracle.  The bound is test_gpu_paged_attention's with its
absolute part: weights below float16's smallest number count nothing."""
import numpy as np
import pytest
import torch

import paper_2601_19675_amd as ptq
from oracle import attention_oracle as orc
from test_gpu_paged_attention import LAYOUTS, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hq,hkv", LAYOUTS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (80, 8), (96, 1), (256, 32), (16, 2), (128, 4), (208, 256)])
def test_layouts(bits, hq, hkv, d, page):
    Problem([75, 37, 300, 64], [75, 17, 33, 1], hq, hkv, d, bits, page, seed=hq * 1000 + d + bits).check(absolute=True, strided=page == 8)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kv,new", [(17, 17), (63, 20), (64, 64), (65, 65), (128, 31), (129, 129), (300, 257), (1000, 18), (5000, 40), (700, 700)])
def test_lengths(bits, kv, new):
    Problem([kv, max(1, kv // 3)], [new, max(1, new // 4)], 4, 2, 64, bits, 16, seed=kv).check(absolute=True)


@pytest.mark.parametrize("d,hq,hkv", [(64, 14, 2), (128, 4, 4), (256, 2, 1)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5), (True, 100), (False, 70), (True, 1)])
def test_masks(d, hq, hkv, causal, window):
    Problem([200, 90, 1500], [130, 90, 20], hq, hkv, d, 8, 16, seed=window).check(causal, window, absolute=True)


def test_more_queries_than_keys_see_nothing():
    Problem([2, 0, 40, 10], [40, 30, 50, 0], 4, 4, 64, 8, 16).check(absolute=True)
    Problem([0, 0], [17, 20], 4, 4, 128, 4, 16).check(absolute=True)


@pytest.mark.parametrize("page", [1, 16, 64])
def test_pages_that_are_not_there(page):
    p = Problem([300, 190, 70], [40, 20, 33], 8, 2, 64, 8, page, seed=page)
    per = p.table.shape[1]
    p.table[0, per // 2], p.table[1, 0], p.table[2, :] = -1, 2 ** 30, -7
    p.check(absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page", [1, 16])
def test_what_is_not_seen_has_no_effect(bits, page):
    p = Problem([61, 130, 47], [20, 1, 47], 4, 2, 64, bits, page, seed=3)
    g = np.random.default_rng(1)
    held = np.zeros(p.scales.shape, dtype=bool)
    for s, c in enumerate(p.kv):
        for j in range(c):
            held[:, p.table[s, j // page], :, j % page] = True
    p.scales[~held] = np.where(g.random((~held).sum()) < 0.5, np.nan, np.inf)
    p.codes[~held] = 255
    p.check(absolute=True)
    p.scales[0, p.table[2, 25 // page], 0, 25 % page] = np.nan
    p.scales[1, p.table[2, 40 // page], 0, 40 % page] = np.nan
    p.scales[1, p.table[0, 60 // page], 1, 60 % page] = np.nan
    p.check(absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("k_size,v_size,q_size", [(1.0, 1e6, 1.0), (1.0, 1e-9, 1.0), (40.0, 1.0, 10.0), (1e-12, 1.0, 1e12), (1e10, 1.0, 1e-10),
                                                  (1e-30, 1.0, 1.0), (1.0, 1e30, 1.0), (1.0, 1e-33, 1.0)])
def test_sizes_of_values(bits, k_size, v_size, q_size):
    p = Problem([513, 60], [20, 40], 8, 4, 64, bits, 16, seed=5, k_size=k_size, v_size=v_size, q_size=q_size)
    p.check(absolute=True)
    # values that grow along the context, by far
    for j in range(513):
        p.scales[1, p.table[0, j // 16], :, j % 16] *= np.float32(2.0 ** (j // 40 - 6))
    p.check(absolute=True)


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_softmax_scales(scale):
    for new in ([1, 2], [20, 40]):
        p = Problem([300, 60], new, 4, 2, 64, 8, 16, seed=9)
        p.scale = scale
        p.check(absolute=True)


def test_queries_of_different_sizes_share_a_tile():
    p = Problem([400, 90], [50, 30], 8, 2, 128, 8, 16, seed=6)
    p.Q = orc.store(p.Q * np.exp2(np.random.default_rng(3).integers(-60, 5, p.Q.shape[:2]))[..., None], "bf16")
    p.Q[0, 3] = 0.0
    p.check(absolute=True)


def test_long_context_of_one_sequence_is_split():
    p = Problem([9000], [33], 4, 1, 128, 8, 64, seed=11)
    p.check(absolute=True)
    p.check(True, 2500, absolute=True)


@pytest.mark.parametrize("bits,d,page", [(8, 128, 16), (4, 64, 16), (8, 256, 32), (4, 80, 1)])
@pytest.mark.parametrize("window", [0, 700])
def test_work_dealt_out_in_shares(bits, d, page, window):
    """Tiles of rows that several workgroups share, others that one has whole, and sequences without queries or keys between them."""
    p = Problem([3000, 700, 0, 5000, 90, 40, 1300], [300, 40, 20, 33, 0, 5, 130], 6, 2, d, bits, page, seed=12)
    p.check(True, window, absolute=True)
    p.check(False, window, absolute=True)


@pytest.mark.parametrize("bits", [8, 4])
def test_pages_missing_and_scales_without_a_value_in_shares(bits):
    p = Problem([5000, 2600], [40, 20], 4, 2, 64, bits, 16, seed=21)
    p.table[0, 10:200] = -1
    p.table[1, :] = 2 ** 30   # nothing there: zeros
    p.check(absolute=True)
    p.scales[1, p.table[0, 4000 // 16], 1, 0] = np.nan
    p.check(absolute=True)


@pytest.mark.parametrize("kv,new", [([4000, 900], [33, 1]), ([700, 650], [700, 600])])
def test_its_stream_and_graph(kv, new):
    p = Problem(kv, new, 8, 2, 128, 8, 16, seed=7)
    want = p.run().clone()
    need = max(256, ptq.ptq_workspace_bytes(ptq.OP_PAGED_ATTENTION, 8, 128, p.Q.shape[0], kv[0]))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(p.run(ws=ws), want)
    dev = lambda a: torch.tensor(a, device="cuda")
    Q = dev(p.Q.astype(np.float32)).bfloat16()
    args = (Q, dev(p.cu), max(new), dev(p.codes), dev(p.scales), dev(p.zeros), 8, dev(p.table), dev(np.array(p.kv, dtype=np.int32)),
            kv[0], p.scale)
    O = torch.zeros_like(Q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ptq.ptq_paged_attention(*args, O, ws=ws)
    for _ in range(3):
        O.zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)
