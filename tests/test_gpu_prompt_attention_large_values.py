"""ptq_prompt_attention on values up to the largest bfloat16: a mean of finite values is finite.  Reference: test_gpu_prompt_attention.  Its bound
counts exponents rounded where they are at most 16 or so; a row whose sums would leave float32's range has them up to 34 further from 0, below 128, rounded to
within 2^-18: weights off by 2^-18 ln 2 more, beside the 2^-8 of their rounding that the bound has, so it is taken 1 + 2^-9 times.  (Weights of less than
2^-92 of such a row's largest may be lost, where it is 2^-126 elsewhere: with scores within 50 of each other there are none.)"""
import math

import pytest
import torch

import paper_2601_19675_amd as ptq
from test_gpu_prompt_attention import BF16, attend, ints, qkv, rand, reference, seen_by, starts

pytestmark = pytest.mark.gpu
MOST = torch.finfo(BF16).max


def held(got, want, bound):
    off, bound = (got.double() - want).abs(), bound * (1 + 2.0 ** -9)
    assert bool(torch.isfinite(got).all()) and bool((off <= bound).all()), (off / bound).max().item()


@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("size", [1e36, 3e37, MOST / 6])     # (six root mean squares: the largest of as many random numbers)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100)])
def test_random_values(d, size, causal, window):
    lengths = [300, 1, 65, 700]
    Q, K, V = qkv(lengths, 4, 2, d, seed=d)
    V = (V.double().clamp(-6, 6) * size).to(BF16)
    held(attend(Q, K, V, lengths, causal=causal, window=window), *reference(Q, K, V, lengths, d ** -0.5, causal, window))


@pytest.mark.parametrize("d", [48, 128, 208])
@pytest.mark.parametrize("q_size", [0.0, 1.0, 4.0])
def test_the_largest_value_everywhere(d, q_size):
    """Means of one number are that number, whatever the weights: a float32 sum of n weights over another order of the same sum, n 2^-24."""
    n = 1500
    Q, K, _ = qkv([n], 2, 1, d, seed=1)
    V = torch.full_like(K, MOST)
    V[:, :, 1::2] = -MOST
    got = attend((Q.float() * q_size).to(BF16), K, V, [n])
    assert torch.equal(got, V.expand_as(got))


@pytest.mark.parametrize("at", [0, 1])
def test_rows_that_do_not_see_them_keep_their_bits(at):
    """Large values in one channel of some tokens, a NaN and an infinity in others, at any address: rows that see none of them are what they were, bit by
    bit, and the others in the channels where none are, but for their exponents' rounding (above)."""
    n, d = 400, 64
    Q, _, _ = qkv([n], 4, 2, d, seed=2)
    flat = torch.empty(2 * (n * 2 * d) + 16, dtype=BF16, device="cuda")
    K, V = (flat[at + i * (n * 2 * d + 8):][:n * 2 * d].view(n, 2, d) for i in range(2))
    K.copy_(rand(n, 2, d, seed=3))
    V.copy_(rand(n, 2, d, seed=4))
    clean = attend(Q, K, V, [n])
    rest, allowed = reference(Q, K, V, [n], d ** -0.5, True, 0)
    V[50:, 0, 3] = 0.9 * MOST
    V[200, 0, 7] = math.nan
    V[230:260, 0, 9] = -math.inf
    got = attend(Q, K, V, [n])
    touched = torch.zeros_like(got, dtype=torch.bool)
    touched[50:, :2, 3] = touched[200:, :2, 7] = touched[230:, :2, 9] = True
    assert torch.equal(got[:50], clean[:50]) and torch.equal(got[:, 2:], clean[:, 2:])
    held(got[~touched], rest[~touched], allowed[~touched])
    assert bool(torch.isnan(got[200:, :2, 7]).all()) and bool((got[230:, :2, 9] == -math.inf).all())
    V[200, 0, 7], V[230:260, 0, 9] = 0.0, 0.0
    want, bound = reference(Q, K, V, [n], d ** -0.5, True, 0)
    held(got[:, :, 3], want[:, :, 3], bound[:, :, 3])


def test_large_values_and_scores_that_grow():
    """The running maximum moves many times while the sums are large."""
    n, d = 900, 128
    Q, K, V = qkv([n], 2, 2, d, seed=5)
    Q = torch.ones_like(Q)
    K = (K.float() * 0.05 + torch.linspace(-0.2, 0.2, n, device="cuda")[:, None, None]).to(BF16)    # scores from -25 to 25
    V = (V.double().clamp(-6, 6) * (MOST / 6)).to(BF16)
    held(attend(Q, K, V, [n], scale=1.0), *reference(Q, K, V, [n], 1.0, True, 0))
    K = K.flip(0).contiguous()
    held(attend(Q, K, V, [n], scale=1.0), *reference(Q, K, V, [n], 1.0, True, 0))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("exponent", [4, 12, 17, 20, 22])
@pytest.mark.parametrize("scale", [1.0, -1.0, 0.75])
def test_scores_up_to_2_30(d, exponent, scale):
    """Scores are whole multiples of 2^exponent up to 256 of them, exactly: a row's mean is that of the tokens with the highest one, whose weights are all
    the same number.  The rest: n others of no more than exp(-|scale| 2^exponent) of it, twice the largest value off; n additions of float32, 2^-14
    of the values' mean size; the output's own rounding, 2^-8."""
    n, g = 700, torch.Generator(device="cuda").manual_seed(exponent)
    Q, K, V = (torch.zeros(n, h, d, dtype=BF16, device="cuda") for h in (2, 1, 1))
    Q[:, :, 5] = 2.0 ** exponent
    k = torch.randint(-256, 257, (n,), device="cuda", generator=g)
    K[:, 0, 5] = k.to(BF16)
    V[:] = rand(n, 1, d, seed=exponent)
    got = attend(Q, K, V, [n], scale=scale).double()
    s = (math.copysign(1, scale) * k).double()[None].expand(n, n).tril() + torch.full((n, n), -1e3, device="cuda").double().triu(1)
    top = (s == s.amax(dim=1, keepdim=True)).double()
    mean = lambda v: (top @ v / top.sum(dim=1, keepdim=True))[:, None]
    want, size = mean(V[:, 0].double()), mean(V[:, 0].double().abs())
    others = n * math.exp(-abs(scale) * 2.0 ** exponent) * 2 * V.double().abs().max()
    assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * want.abs() + 2.0 ** -14 * size + others).all())


def test_keys_that_are_not_numbers_beside_large_values():
    n, d = 200, 64
    Q, K, V = (x.contiguous() for x in qkv([n], 1, 1, d, seed=6))
    V = (V.double().clamp(-6, 6) * (MOST / 6)).to(BF16)
    K[120, 0, 0] = math.nan
    got = attend(Q, K, V, [n])
    want, bound = reference(Q[:120], K[:120], V[:120], [120], d ** -0.5, True, 0)
    held(got[:120], want, bound)
    assert bool(torch.isnan(got[120:]).all())
