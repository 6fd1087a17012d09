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


def one(name, args, read):
    (rc, launches), = record([(name, args)], read=read)
    assert rc == OK and launches
    return launches


@pytest.mark.parametrize("t,n,dt,threads", [(2 ** 25 + 5, 4096, 1, 256), (2 ** 27 + 1, 64, 0, 256), (2 ** 22 + 3, 32768, 1, 1024), (1000, 4096, 1, 256)])
def test_norm_of_many_rows(t, n, dt, threads):
    size = 2 if dt == 1 else 4
    args = [PTR, dt, n, t, n, 2 * PTR, n + 8, 3 * PTR, n + 16, PTR, 1e-5, 1, 4 * PTR, n + 32, 5 * PTR, 0]
    fields = dict(X=(0, "q", 0), R=(0, "q", 8), Y=(0, "q", 16), C=(0, "q", 32), S=(0, "q", 40), t=(0, "i", 80))
    done = 0
    for k in one("ptq_rmsnorm_quantize", args, {"rmsnorm_quantize_kernel": fields}):
        assert 0 < k["grid"][0] * threads < THREADS and k["grid"][1:] == [1, 1]
        assert k["grid"][0] >= (k["t"] if n > 2048 else -(-k["t"] // 4))
        assert (k["X"], k["R"], k["Y"]) == (PTR + done * n * size, 2 * PTR + done * (n + 8) * size, 3 * PTR + done * (n + 16) * size)
        assert (k["C"], k["S"]) == (4 * PTR + done * (n + 32), 5 * PTR + 4 * done)
        done += k["t"]
    assert done == t


@pytest.mark.parametrize("t,hkv,d", [(2 ** 26 + 9, 32, 128), (2 ** 25, 32767, 16), (1000, 8, 128), (2 ** 30 - 1, 64, 256)])
def test_cache_write_of_many_tokens(t, hkv, d):
    args = [PTR, hkv * d, d, 2 * PTR, hkv * d + 16, d, 1, t, hkv, d, 3 * PTR, 8, PTR, PTR, PTR, 8, 16, 0]
    fields = dict(K=(0, "q", 0), V=(0, "q", 8), slots=(0, "q", 48), t=(0, "i", 56))
    per = 4 * 256 // (8 if d <= 64 else 16 if d <= 128 else 32)
    done = 0
    for k in one("ptq_kv_cache_write", args, {"kv_write_kernel": fields}):
        assert 0 < k["grid"][0] * 256 < THREADS and k["grid"][1:] == [2, 1] and k["grid"][0] == -(-k["t"] // per) * hkv
        assert (k["K"], k["V"], k["slots"]) == (PTR + 2 * done * hkv * d, 2 * PTR + 2 * done * (hkv * d + 16), 3 * PTR + 4 * done)
        done += k["t"]
    assert done == t


@pytest.mark.parametrize("max_kv,rows,hkv,d", [(2 ** 30 - 1, 2 ** 29, 32, 64), (2 ** 30 - 1, 2 ** 30, 32767, 16), (2 ** 30 - 1, 1000, 8, 128), (700, 5000, 8, 128),
                                               (2 ** 30 - 1, 1, 32767, 256)])
def test_cache_read_of_long_sequences(max_kv, rows, hkv, d):
    args = [PTR, PTR, PTR, 8, 16, hkv, d, 8, PTR, 4, 3, PTR, rows, max_kv, PTR, hkv * d, d, PTR, hkv * d, d, 1, 0]
    per = 4 * 256 // (8 if d <= 64 else 16 if d <= 128 else 32)
    done = 0   # tiles of places of a sequence
    for k in one("ptq_kv_cache_read", args, {"kv_read_kernel": dict(first=(0, "i", 92))}):
        assert 0 < k["grid"][0] * 256 < THREADS and k["grid"][1:] == [2, 3] and k["grid"][0] % hkv == 0 and k["first"] == done
        done += k["grid"][0] // hkv
    # max_kv is a bound: no sequence has more places than there are rows
    assert done == -(-min(max_kv, rows) // per)


@pytest.mark.parametrize("b,hq,hkv,max_q,d", [(4096, 32, 32, 2 ** 17, 64), (65535, 8, 8, 300, 64), (3, 8, 1, 2 ** 24, 64), (9, 8, 2, 300, 256), (65535, 32767, 32767, 17, 16)])
def test_chunks_of_many_sequences(b, hq, hkv, max_q, d):
    t = 2 ** 24
    args = attention(t, hq, hkv, max_q, b=b, max_kv=1000, ws=PTR)
    args[6] = d
    threads, rows = (256, 128) if d > 128 else (512, 256)
    tiles = -(-max_q * (hq // hkv) // rows)
    done = 0   # groups: a sequence and a key head each, eight side by side
    for k in one("ptq_paged_attention", args, {"attend_chunk_kernel": dict(tiles=(1, "i"), first=(2, "i"))}):
        assert 0 < k["grid"][0] * threads < THREADS and k["grid"][1:] == [1, 1]
        assert k["tiles"] == tiles and k["first"] == done and k["grid"][0] % (8 * tiles) == 0
        done += k["grid"][0] // tiles
    assert b * hkv <= done < b * hkv + 8


@pytest.mark.parametrize("scale,status", [(1e39, 1), (-1e300, 1), (2.4e38, 1), (3e37, WORKSPACE), (0.0, WORKSPACE)])
def test_softmax_scales_that_float32_does_not_hold(scale, status):
    args = attention(4, 8, 2, 3)
    args[21] = scale
    (rc, launches), = record([("ptq_paged_attention", args)])
    assert rc == status and not launches
