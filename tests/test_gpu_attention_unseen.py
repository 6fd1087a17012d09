"""A key that a query does not see has no effect on its row, however large or small what it holds: rows that do not see an altered key keep
every bit, rows that see it follow the float64 oracle, with a bound that knows only the keys that a row sees."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as orc
from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu

FACTORS = [2.0 ** 20, 2.0 ** 40, 1e30, 2.0 ** -25, 2.0 ** -60]


def seen_keys(p, s, causal, window):
    """[new, kv] of sequence s."""
    length, new = p.kv[s], p.new[s]
    place, j = length - new + np.arange(new)[:, None], np.arange(length)[None]
    sees = np.ones((new, length), dtype=bool)
    if causal:
        sees &= j <= place
    if window:
        sees &= j > place - window
    return sees


def check_seen(p, got, causal, window):
    """The bound of Problem.check, its absolute part with the largest value that the row itself sees: a weight below float16's normal numbers is
    off by 2^-25, of a unit that the largest weight is half of or more, and the value of such a key may be brought to twice the largest's
    place in float16's range; a grid may have its zero at one end (a factor of two between a scale and its largest value): 2^-22."""
    got = got.double().cpu().numpy()
    want, size, reach = orc.attention(p.Q, p.cu, p.codes, p.scales, p.zeros, p.bits, p.table, p.kv, p.scale, causal, window, spread=True)
    rel = 3 * 2.0 ** -11 + 2 * ((p.d + 8) * 2.0 ** -24 * reach[..., None] + 2.0 ** -21)
    tol = 2.0 ** -8 * np.abs(want) * 1.01 + rel * size + 2.0 ** -133
    largest = np.abs(p.scales[1].astype(np.float64)) * np.maximum(p.zeros[1], 2 ** p.bits - 1 - p.zeros[1].astype(np.int64))
    page, group = p.scales.shape[3], p.hq // p.scales.shape[2]
    for s, length in enumerate(p.kv):
        sees = seen_keys(p, s, causal, window)
        j = np.arange(length)
        held = largest[p.table[s, j // page], :, j % page]                        # [kv, heads]
        top = np.where(sees[:, :, None], held[None], 0.0).max(1)                  # [new, heads]
        tol[p.cu[s]:p.cu[s + 1]] += (sees.sum(1)[:, None] * 2.0 ** -22 * top).repeat(group, 1)[..., None]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])


def altered(p, s, places, factor, keys_too):
    """Multiplies the value scales of these places, and the key scales of those that nobody is to see."""
    page = p.scales.shape[3]
    j = np.asarray(places)
    p.scales[1, p.table[s, j // page], :, j % page] *= np.float32(factor)
    if keys_too:
        p.scales[0, p.table[s, j // page], :, j % page] *= np.float32(factor)


def both(kv, new, hq, hkv, d, bits, page, s, places, factor, causal=True, window=0, keys_too=False):
    p = Problem(kv, new, hq, hkv, d, bits, page, seed=d + bits + len(places))
    before = p.run(causal, window)
    check_seen(p, before, causal, window)
    altered(p, s, places, factor, keys_too)
    after = p.run(causal, window)
    sees = seen_keys(p, s, causal, window)[:, places].any(1)
    keeps = np.ones(p.Q.shape[0], dtype=bool)
    keeps[p.cu[s]:p.cu[s + 1]] = ~sees
    assert keeps.any()
    keeps = torch.tensor(keeps, device="cuda")
    assert torch.equal(after[keeps], before[keeps])
    check_seen(p, after, causal, window)


@pytest.mark.parametrize("factor", FACTORS)
@pytest.mark.parametrize("bits,d,page", [(8, 128, 16), (4, 64, 32), (8, 256, 16), (4, 80, 4)])
def test_keys_below_the_window(bits, d, page, factor):
    # the first query sees keys from 181 on; its tile of 64 begins at 128
    both([300, 50], [20, 3], 8, 2, d, bits, page, 0, list(range(100, 181)), factor, window=100, keys_too=True)


@pytest.mark.parametrize("factor", FACTORS)
@pytest.mark.parametrize("bits,d,page", [(8, 128, 16), (4, 128, 64), (8, 64, 16), (4, 256, 32), (8, 96, 1)])
def test_later_tokens_of_a_chunk(bits, d, page, factor):
    both([150, 40], [150, 40], 4, 2, d, bits, page, 0, [90, 91, 140], factor)
    both([150, 40], [150, 40], 4, 2, d, bits, page, 0, [3], factor)


@pytest.mark.parametrize("factor", FACTORS)
@pytest.mark.parametrize("bits,d", [(8, 128), (4, 64)])
def test_later_tokens_where_work_is_shared(bits, d, factor):
    both([5000, 2600], [300, 40], 4, 2, d, bits, 16, 0, [4800, 4990], factor)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new", [[60, 1]])
def test_values_of_every_size(bits, new):
    """Value scales from 2^-100 to 2^80 side by side, most of them far from the row's largest."""
    p = Problem([700, 33], new, 8, 2, 64, bits, 16, seed=13)
    p.scales[1] *= np.exp2(np.random.default_rng(4).integers(-100, 80, p.scales[1].shape)).astype(np.float32)
    check_seen(p, p.run(), True, 0)
    # a context that is small throughout, and one that grows small along its keys
    p = Problem([700, 33], new, 8, 2, 64, bits, 16, seed=14, v_size=1e-20)
    check_seen(p, p.run(), True, 0)
    p = Problem([700, 33], new, 8, 2, 64, bits, 16, seed=15)
    for j in range(700):
        p.scales[1, p.table[0, j // 16], :, j % 16] *= np.float32(2.0 ** -(j // 10))
    check_seen(p, p.run(), True, 0)
