"""A query stands at place kv_lens - new + i also where the page table or max_kv ends before the sequence does: keys past them are not there, and
nothing else moves."""
import numpy as np
import pytest
import torch

import paper_2601_19675_amd as ptq
from oracle import attention_oracle as orc
from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,new", [([700, 300], [1, 1]), ([300, 90], [4, 2]), ([300, 90], [100, 40]), ([5000, 4200], [1, 1]), ([5000, 90], [60, 40])])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 90), (False, 60), (False, 0)])
@pytest.mark.parametrize("cut", ["table", "max_kv"])
def test_places_do_not_move(kv, new, causal, window, cut):
    p = Problem(kv, new, 8, 2, 64, 8, 16, seed=41)
    there = 16 * (kv[0] // 20)            # keys that are left, of every sequence
    table = p.table[:, : there // 16].copy()
    dev = lambda a: torch.tensor(a, device="cuda")
    Q = dev(p.Q.astype(np.float32)).bfloat16()
    O = torch.full_like(Q, 5.0)
    ptq.ptq_paged_attention(Q, dev(p.cu), max(new), dev(p.codes), dev(p.scales), dev(p.zeros), 8, dev(table if cut == "table" else p.table),
                            dev(np.array(kv, dtype=np.int32)), max(kv) if cut == "table" else there, p.scale, O, causal=causal, window=window)
    got = O.double().cpu().numpy()
    want, size, reach = orc.attention(p.Q, p.cu, p.codes, p.scales, p.zeros, 8, table, kv, p.scale, causal, window, spread=True)
    # the bound of Problem.check, with its absolute part; values are of one size here
    top = (p.scales[1].astype(np.float64) * np.maximum(p.zeros[1], 255 - p.zeros[1].astype(np.int64))).max()
    rel = 3 * 2.0 ** -11 + 2 * ((p.d + 8) * 2.0 ** -24 * reach[..., None] + 2.0 ** -21)
    tol = 2.0 ** -8 * np.abs(want) * 1.01 + rel * size + there * 2.0 ** -24 * top + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])
