"""What the calls of the 8-bit attention path do with more rows than a launch or 32 bits hold (no GPU: refusals, and the launches that the recording
stand-in for the runtime sees)."""
import pytest

import paper_2601_19675_amd as ptq
from launch_recorder import PTR, record

OK, SHAPE, WORKSPACE = 0, 2, 4
THREADS = 2 ** 32   # of a launch, in one direction, fewer than that


def attention(t, hq, hkv, max_q, b=2, max_kv=5000, ws=0):
    return [PTR, 1, 64 * hq, 64, t, hq, 64, PTR, b, max_q, PTR, PTR, PTR, 8, 16, hkv, 8, PTR, 2, PTR, max_kv, 0.125, 1, 0, 2 * PTR, 64 * hq, 64, ws,
            2 ** 60, 0]


def test_query_rows_of_a_key_head():
    # 2^27 of them, tokens times group: what the chunks' tiles are counted in
    calls = [attention(2 ** 24, 16, 1, 2 ** 24), attention(2 ** 24, 128, 1, 2 ** 24), attention(2 ** 24, 65535, 1, 2 ** 24),
             attention(2 ** 24, 8, 1, 2 ** 24), attention(2 ** 24, 128, 1, 2 ** 20)]
    got = [rc for rc, _ in record([("ptq_paged_attention", a) for a in calls])]
    assert got == [SHAPE, SHAPE, SHAPE, WORKSPACE, WORKSPACE]
