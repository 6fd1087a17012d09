"""Pins of the 8-bit attention path's oracle: values worked out by hand, and identities that the definitions imply."""
import numpy as np
import pytest

from oracle import attention_oracle as orc


def test_norm_by_hand():
    # rms of (3, 4) is sqrt(12.5); the largest becomes 127, the other 95.25 -> 95
    codes, scales, y = orc.rmsnorm_quantize([[3.0, -4.0]], eps=0.0)
    assert codes.tolist() == [[95, -127]] and abs(scales[0] - 4 / 127 / np.sqrt(12.5)) < 1e-15
    # a tie goes to the even code: 254 u / A = 2 k + 1 with A = 254, u = 0.5, 1.5
    codes, _, _ = orc.rmsnorm_quantize([[127.0 * 2, 1.0, 3.0, -1.0]], normalize=False)
    assert codes.tolist() == [[127, 0, 2, 0]]
    codes, scales, _ = orc.rmsnorm_quantize([[0.0, 0.0], [1.0, np.inf]])
    assert not codes.any() and scales[0] == 0 and np.isnan(scales[1])
    # the sum is rounded to the storage type before anything else
    _, _, y = orc.rmsnorm_quantize([[256.0, 1.0]], dtype="bf16", residual=[[1.0, 0.0]])
    assert y.tolist() == [[256.0, 1.0]]


def test_row_grid_by_hand():
    codes, scale, zero = orc.quantize_row([-1.0, 0.0, 2.0, 0.5], 4)
    assert scale == np.float32(0.2) and zero == 5 and codes.tolist() == [0, 5, 15, 7]
    codes, scale, zero = orc.quantize_row(np.zeros(4), 8)
    assert scale == np.float32(2 / 255) and (codes == zero).all()
    assert np.isnan(orc.quantize_row([1.0, np.nan], 8)[1])


@pytest.mark.parametrize("bits", [4, 8])
def test_packing(bits):
    codes = np.arange(32) % 2 ** bits
    assert (orc.unpack_row(orc.pack_row(codes, bits), bits) == codes).all()
    if bits == 4:   # codes 0 .. 7: even ones in the low half word, odd ones in the high
        assert orc.pack_row(np.arange(8), 4).view("<u4")[0] == 0x75316420


def test_attention_identities():
    g = np.random.default_rng(1)
    t, hkv, d, page = 9, 2, 16, 4
    K, V = g.standard_normal((t, hkv, d)), g.standard_normal((t, hkv, d))
    cache = (np.zeros((2, 4, hkv, page, d), np.uint8), np.zeros((2, 4, hkv, page), np.float32), np.zeros((2, 4, hkv, page), np.uint8))
    table = np.array([[2, 0, 3]])
    slots = [table[0][i // page] * page + i % page for i in range(t)]
    orc.cache_write(K, V, slots, 8, *cache)
    back, there = orc.cache_rows(*cache, 8, table[0], t, 1)
    assert there.all() and np.abs(back - V).max() < 0.02
    Q = g.standard_normal((1, 4, d))
    # the last token sees everything; with a window of one it sees its own value row only
    O = orc.attention(Q, [0, 1], *cache, 8, table, [t], 0.25, window=1)
    assert np.allclose(O[0], back[t - 1][[0, 0, 1, 1]])
    # no softmax scale: the mean of the values; more queries than keys: the first see nothing
    assert np.allclose(orc.attention(Q, [0, 1], *cache, 8, table, [t], 0.0)[0], back.mean(0)[[0, 0, 1, 1]])
    O = orc.attention(np.repeat(Q, 3, 0), [0, 3], *cache, 8, table, [2], 0.25)
    assert not O[0].any() and np.allclose(O[1], back[0][[0, 0, 1, 1]])
    # a page that is not there is not seen
    O = orc.attention(Q, [0, 1], *cache, 8, np.array([[2, -1, 3]]), [t], 0.0)
    assert np.allclose(O[0], back[[0, 1, 2, 3, 8]].mean(0)[[0, 0, 1, 1]])
