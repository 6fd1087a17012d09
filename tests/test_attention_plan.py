"""Whether attention of chunks lays its work out in shares, by sizes (no GPU: the runtime is the recording stand-in).  Tiles of 256 rows (128 beyond
128 channels), one workgroup to a compute unit, 256 of them."""
import pytest

from launch_recorder import PTR, record


def shared(b, t, max_q, max_kv, hq=32, hkv=8, d=128, window=0):
    args = [PTR, 1, d * hq, d, t, hq, d, PTR, b, max_q, PTR, PTR, PTR, 8, 16, hkv, 8, PTR, 2, PTR, max_kv, 0.125, 1, window, 2 * PTR, d * hq, d, PTR,
            2 ** 60, 0]
    (rc, launches), = record([("ptq_paged_attention", args)])
    assert rc == 0 and "attend_chunk_kernel" in launches[0]["kernel"]
    return any("join_chunk_kernel" in k["kernel"] for k in launches)


@pytest.mark.parametrize("want,case", [
    (False, dict(b=3, t=3 * 2048, max_q=2048, max_kv=8192)),       # 768 tiles: three full rounds
    (False, dict(b=2, t=2 * 2048, max_q=2048, max_kv=16384)),
    (True, dict(b=2, t=2048 + 1035, max_q=2048, max_kv=16384)),     # 400 tiles at most, by the tokens there are
    (True, dict(b=1, t=2048, max_q=2048, max_kv=16384)),            # one round: contexts may differ
    (False, dict(b=1, t=2048, max_q=2048, max_kv=2048)),
    (True, dict(b=1, t=64, max_q=64, max_kv=2048)),
    (False, dict(b=1, t=64, max_q=64, max_kv=1024)),                # too short for a second kernel
    (True, dict(b=9, t=1024 + 8, max_q=1024, max_kv=32768)),        # a chunk beside single tokens: 200 tiles, not 1152
    (True, dict(b=64, t=512 + 63, max_q=512, max_kv=32768)),
    (False, dict(b=9, t=2400, max_q=300, max_kv=5000, hq=28, hkv=4, d=64, window=1024)),
    (True, dict(b=9, t=1600, max_q=300, max_kv=5000, hq=28, hkv=4, d=64)),
    (False, dict(b=1, t=2 ** 20, max_q=2 ** 20, max_kv=2 ** 20)),   # more rounds than need it
])
def test_shares(want, case):
    assert shared(**case) == want
