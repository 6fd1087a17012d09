"""ptq_prompt_attention against softmax attention in float64.

Bound of an output, with p the weights: a weight is rounded to bfloat16, 2^-8 of itself, and its score s is off by e: d + 2 additions and
products of float32 in softmax_scale sum |q| |k|, and the exponent's argument, no further from 0 than |s| + 8 log2(e), by two roundings.  The
sum of the weights is of the rounded ones, so a relative error of the weights moves the mean by at most that times sum p |v - O| / sum p, no more than
2 sum p |v| / sum p.  The sums themselves: n additions of float32, sqrt(n) of them at once in the worst of orders here (n / 16 + 20).  Then the
output's own rounding, 2^-8."""
import math

import pytest
import torch

import paper_2601_19675_amd as ptq

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def rand(*shape, seed=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn(*shape, device="cuda", generator=g)).to(BF16)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def seen_by(n, causal, window):
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    see = torch.ones(n, n, dtype=torch.bool, device="cuda")
    if causal:
        see &= j <= i
    if window:
        see &= j > i - window
    return see


def reference(Q, K, V, lengths, scale, causal, window):
    """(output, bound) in float64, on the device."""
    out, bound = torch.zeros(Q.shape, dtype=torch.float64, device="cuda"), torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    group, d = Q.shape[1] // K.shape[1], Q.shape[2]
    for a, n in zip(starts(lengths), lengths):
        see = seen_by(n, causal, window)
        for h in range(Q.shape[1]):
            q, k, v = Q[a:a + n, h].double(), K[a:a + n, h // group].double(), V[a:a + n, h // group].double()
            s = (scale * (q @ k.T.contiguous())).masked_fill(~see, -math.inf)
            p = s.softmax(dim=1)
            o = p @ v
            reach = abs(scale) * (q.abs() @ k.abs().T.contiguous()).masked_fill(~see, 0.0).amax(dim=1, keepdim=True)
            e = (d + 6) * 2.0 ** -24 * reach + 16 * 2.0 ** -24
            size = p @ v.abs()
            out[a:a + n, h] = o
            bound[a:a + n, h] = 2.0 ** -8 * o.abs() + 2 * (2.0 ** -8 + 2 * e + (n / 16 + 20) * 2.0 ** -24) * size * (1 + 2.0 ** -7)
    return out, bound


def attend(Q, K, V, lengths, scale=None, causal=True, window=0, O=None, max_n=None):
    O = torch.full_like(Q, 7.0, memory_format=torch.contiguous_format) if O is None else O
    ptq.ptq_prompt_attention(Q, K, V, ints(starts(lengths)), max(lengths) if max_n is None else max_n, Q.shape[2] ** -0.5 if scale is None else scale, O,
                             causal=causal, window=window)
    return O


def check(Q, K, V, lengths, scale=None, causal=True, window=0):
    scale = Q.shape[2] ** -0.5 if scale is None else scale
    got = attend(Q, K, V, lengths, scale, causal, window)
    want, bound = reference(Q, K, V, lengths, scale, causal, window)
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (off / bound).max().item()
    # the two roundings are independent ones of any sign: together below a whole step of the root mean square
    assert ((got.double() - want).norm() <= 2.0 ** -8 * want.norm() + 1e-30).item() or max(lengths) < 8
    return got


def qkv(lengths, hq, hkv, d, seed=0, size=1.0):
    all_ = rand(sum(lengths), hq + 2 * hkv, d, seed=seed, size=size)
    return all_.split([hq, hkv, hkv], dim=1)


@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (7, 1), (14, 2), (3, 3), (1, 1)])
@pytest.mark.parametrize("d", [16, 64, 80, 96, 112, 128, 208, 256])
def test_layouts(hq, hkv, d):
    lengths = [75, 1, 130, 64, 33]
    check(*qkv(lengths, hq, hkv, d, seed=hq * 1000 + d), lengths)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 300, 511, 512, 513, 700, 1023, 1025])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_lengths(n, d):
    lengths = [n, max(1, n // 3)]
    check(*qkv(lengths, 4, 2, d, seed=n), lengths)
    check(*qkv(lengths, 2, 2, d, seed=n), lengths, causal=False)


@pytest.mark.parametrize("d,hq,hkv", [(64, 7, 1), (96, 2, 2), (128, 4, 1), (256, 3, 3)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 5), (True, 64), (True, 100), (False, 1), (False, 70), (True, 10 ** 9)])
def test_which_tokens_a_row_sees(d, hq, hkv, causal, window):
    """Scores of 0 and values of one channel each: an output counts the tokens of its channel, with nothing but its own rounding."""
    lengths = [200, 1, 63, 517, 128]
    t = sum(lengths)
    Q, K = torch.zeros(t, hq, d, dtype=BF16, device="cuda"), rand(t, hkv, d, seed=1)
    V = torch.zeros(t, hkv, d, device="cuda")
    for a, n in zip(starts(lengths), lengths):
        for h in range(hkv):
            V[a:a + n, h] = torch.eye(d, device="cuda")[(torch.arange(n, device="cuda") + h) % d]
    got = attend(Q, K, V.to(BF16), lengths, causal=causal, window=window).double()
    for a, n in zip(starts(lengths), lengths):
        see = seen_by(n, causal, window).double()
        for h in range(hq):
            want = see @ V[a:a + n, h // (hq // hkv)].double() / see.sum(dim=1, keepdim=True)
            assert bool(((got[a:a + n, h] - want).abs() <= 2.0 ** -8 * want + 2.0 ** -22 * want).all())


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0, 1e-30])
def test_softmax_scales(scale):
    lengths = [300, 41]
    check(*qkv(lengths, 4, 2, 64, seed=9, size=0.3), lengths, scale=scale)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_size,v_size", [(30.0, 1.0), (1e-20, 1.0), (1.0, 1e30), (1.0, 1e-30), (100.0, 1e5)])
def test_sizes(d, q_size, v_size):
    lengths = [333, 70]
    Q, K, V = qkv(lengths, 4, 2, d, seed=5)
    got = attend((Q.float() * q_size).to(BF16), K, (V.float() * v_size).to(BF16), lengths).double()
    want, bound = reference((Q.float() * q_size).to(BF16), K, (V.float() * v_size).to(BF16), lengths, d ** -0.5, True, 0)
    assert bool(((got - want).abs() <= bound).all())


def test_scores_that_rise_and_fall_by_far():
    """The running maximum moves late, early, and back: keys that grow along the prompt, shrink, or alternate."""
    n, d = 600, 64
    Q, K, V = qkv([n], 2, 2, d, seed=6)
    ramp = torch.linspace(-60, 60, n, device="cuda")
    for shape in (ramp, -ramp, 40 * torch.sin(ramp)):
        K2 = (0.1 * K.float() + 0.125 * Q.float().mean(dim=(0, 1)) + shape[:, None, None] * torch.sign(Q[n // 2].float()) / d).to(BF16)
        check(Q, K2, V, [n], scale=1.0)
        check(Q, K2, V, [n], scale=1.0, causal=False)


@pytest.mark.parametrize("d", [80, 128, 240])
def test_strides_and_addresses(d):
    """Rows at odd addresses, heads before tokens, gaps between rows, one key head for all tokens' heads; what lies between is left alone."""
    lengths, hq, hkv = [70, 5, 129], 6, 2
    t = sum(lengths)
    Q, K, V = (x.contiguous() for x in qkv(lengths, hq, hkv, d, seed=d))
    want = attend(Q, K, V, lengths)

    def moved(x, pitch, head, at):
        flat = torch.full((at + t * pitch + 8,), float("nan"), dtype=BF16, device="cuda")
        y = flat[at:].as_strided(x.shape, (pitch, head, 1))
        y.copy_(x)
        return flat, y
    for at, odd in ((0, 0), (1, 0), (8, 3), (3, 8)):
        _, q = moved(Q, hq * (d + 3), d + 3, at)
        _, k = moved(K, hkv * (d + 8) + odd, d + 8, at)
        _, v = moved(V, hkv * d + 24, d, at)
        flat, o = moved(Q, hq * (d + 5) + 1, d + 5, 3)
        o.fill_(1.0)
        before = flat.clone()
        attend(q, k, v, lengths, O=o)
        assert torch.equal(o, want), (at, odd)
        o.fill_(1.0)
        assert torch.equal(flat.view(torch.int16), before.view(torch.int16))
    heads_first = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (Q, K, V)]
    assert torch.equal(attend(*heads_first, lengths), want)
    one = K[:, :1].expand(t, 3, d), V[:, :1].expand(t, 3, d)     # a head stride of 0
    assert torch.equal(attend(Q, *one, lengths), attend(Q, one[0].contiguous(), one[1].contiguous(), lengths))
    assert torch.equal(attend(Q, K, V, lengths, O=Q), want)      # in place


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (2, 2, 64), (2, 1, 256)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 40), (False, 40), (False, 0)])
def test_what_is_not_seen_has_no_effect(hq, hkv, d, causal, window):
    """Infinities, NaN and the largest numbers in tokens that a row does not see -- later ones, those before its window, other prompts', those
    of nobody -- leave it as it is, bit by bit; in tokens that it sees they reach the channels that they are in."""
    lengths = [150, 20, 97]
    Q, K, V = (x.contiguous() for x in qkv(lengths, hq, hkv, d, seed=3))
    clean = attend(Q, K, V, lengths, causal=causal, window=window)
    for spot, what in ((60, float("nan")), (149, float("inf")), (0, -float("inf")), (151, float("nan")), (200, 3e38), (266, float("nan"))):
        a, n = next((a, n) for a, n in zip(starts(lengths), lengths) if a <= spot < a + n)
        reached = torch.zeros(Q.shape[0], dtype=torch.bool, device="cuda")
        reached[a:a + n] = seen_by(n, causal, window)[:, spot - a]
        V2 = V.clone()
        V2[spot, 0, 5] = what
        got = attend(Q, K, V2, lengths, causal=causal, window=window)
        heads = torch.arange(hq, device="cuda") < hq // hkv
        touched = torch.zeros_like(Q, dtype=torch.bool)
        touched[:, :, 5] = reached[:, None] & heads
        assert torch.equal(got[~touched], clean[~touched]), spot
        if not math.isfinite(what):
            bad = got[touched]
            assert bool(torch.isnan(bad).all() if math.isnan(what) else (bad == what).all())
        K2 = K.clone()
        K2[spot, 0] = what if math.isfinite(what) else float("nan")
        got = attend(Q, K2, V, lengths, causal=causal, window=window)
        touched = (reached[:, None] & heads)[:, :, None].expand_as(got)
        assert torch.equal(got[~touched], clean[~touched]), spot
        if not math.isfinite(what):
            assert bool(torch.isnan(got[touched]).all())
    Q2 = Q.clone()
    Q2[70, 1] = float("nan")
    got = attend(Q2, K, V, lengths, causal=causal, window=window)
    rest = torch.ones_like(Q, dtype=torch.bool)
    rest[70, 1] = False
    assert torch.equal(got[rest], clean[rest]) and bool(torch.isnan(got[70, 1]).all())


def test_opposite_infinities_that_are_seen_are_nan():
    Q, K, V = (x.contiguous() for x in qkv([40], 1, 1, 64, seed=4))
    V[3, 0, 9], V[11, 0, 9], V[20, 0, 2] = float("inf"), -float("inf"), float("inf")
    got = attend(Q, K, V, [40])
    assert bool(torch.isfinite(got[:3]).all()) and bool((got[3:11, 0, 9] == float("inf")).all()) and bool(torch.isnan(got[11:, 0, 9]).all())
    assert bool((got[20:, 0, 2] == float("inf")).all())
    odd = torch.zeros_like(got, dtype=torch.bool)
    odd[3:, 0, 9] = odd[20:, 0, 2] = True
    assert bool(torch.isfinite(got[~odd]).all())


def test_prompts_that_do_not_fit_and_rows_of_nobody():
    Q, K, V = (x.contiguous() for x in qkv([100], 2, 1, 64, seed=8))
    O = torch.full_like(Q, 7.0)
    call = lambda cu, max_n: ptq.ptq_prompt_attention(Q, K, V, ints(cu), max_n, 0.125, O)
    call([-5, 10, 40, 40, 101], 100)      # begins before token 0; fits; is empty; ends past the last
    want = torch.full_like(Q, 7.0)
    want[10:40] = attend(Q[10:40], K[10:40], V[10:40], [30])
    assert torch.equal(O, want)
    O.fill_(7.0)
    call([10, 90], 37)                    # longer than max_n says: the tokens from there on are left out
    want.fill_(7.0)
    want[10:47] = attend(Q[10:47], K[10:47], V[10:47], [37])
    assert torch.equal(O, want)
    O.fill_(7.0)
    ptq.ptq_prompt_attention(Q, K, V, ints([10, 90]), 37, 0.125, O, causal=False)
    want[10:47] = attend(Q[10:47], K[10:47], V[10:47], [37], causal=False)
    assert torch.equal(O, want)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_a_long_prompt_among_short_ones(hq, hkv, d):
    lengths = [9, 2500, 300, 1, 700]
    got = check(*qkv(lengths, hq, hkv, d, seed=10), lengths)
    Q, K, V = qkv(lengths, hq, hkv, d, seed=10)
    a = starts(lengths)
    for s in (0, 1, 2, 4):   # the same, whatever lies beside it
        own = slice(a[s], a[s + 1])
        assert torch.equal(attend(Q[own], K[own], V[own], [lengths[s]]), got[own])
    assert torch.equal(attend(Q, K, V, lengths, max_n=sum(lengths)), got)


def test_replayed_and_on_another_stream():
    t, hq, hkv, d = 400, 4, 2, 128
    Q, K, V = qkv([t], hq, hkv, d, seed=1)
    cu, O = ints([0, 300, 400, 400]), torch.zeros(t, hq, d, dtype=BF16, device="cuda")
    call = lambda: ptq.ptq_prompt_attention(Q, K, V, cu, 400, d ** -0.5, O)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, ends in enumerate(([0, 300, 400, 400], [0, 1, 2, 400], [0, 0, 400, 400], [0, 130, 270, 400])):
        cu.copy_(ints(ends))
        Q.copy_(rand(t, hq, d, seed=20 + i))
        graph.replay()
        got = O.clone()
        O.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(O, got), i
        check(Q, K, V, [b - a for a, b in zip(ends, ends[1:]) if b > a])
