"""Performance cases of what stands around the paged quantized cache: rotary positions, alone and on the way into the cache,
pages copied when sequences fork or a cache is compacted, attention of sequences that share a prefix, and attention of
whole prompts before their keys and values are quantized.

Sizes are those of the benchmark's configurations (32 heads of 128 channels) and generic ones beside them: shared
key heads, head widths of 64 to 256, pages of 1 to 256 tokens.

With `own` false every operator is computed by elementary torch operations in float32 (angles, rotations and grids in
float64, whose roundings decide codes); with `own` true by the library's calls.  `exact` restates them in float64.

The cache: codes [2, pages, heads, page, width bits / 8], scales and zeros [2, pages, heads, page]; index 0 holds the keys, 1
the values.  A code c stands for scale (c - zero).  8 bits: a byte per code.  4 bits: eight codes make a little-endian 32-bit
word, code 2 i of them in bits 4 i and code 2 i + 1 in bits 16 + 4 i.
"""
from __future__ import annotations

import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


# ---------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # Queries and keys of sixteen sequences' next tokens, turned in the projection's output before both go on: all latency.
        dict(name="rotary_decode_16", kind="rotary", t=16, heads=40, d=128, rot=128, interleaved=False, dtype="bf16", factor=1.0, far=30000),
        # Queries and keys of long prompts at frequencies that are slowed for long contexts: bytes.
        dict(name="rotary_prompt_16384", kind="rotary", t=16384, heads=40, d=128, rot=128, interleaved=True, dtype="bf16", factor=8.0, far=131072),
        # Sixteen sequences' next tokens turned and put into the cache, whose short contexts then move on.
        dict(name="rotary_cache_decode_16", kind="into", b=16, kv=211, new=1, hq=32, hkv=8, d=128, rot=128, interleaved=False, bits=8, page=16,
             dtype="bf16", factor=1.0),
        # Prompts enter a 4-bit cache, half of a head's channels turned, and move on.
        dict(name="rotary_cache_prompt", kind="into", b=4, kv=4096, new=4096, hq=32, hkv=32, d=128, rot=64, interleaved=False, bits=4, page=64,
             dtype="bf16", factor=4.0),
        # The last pages of 24 forks of a sequence: latency.
        dict(name="copy_fork_24", kind="copy", n=24, pages=700, hkv=8, d=128, bits=8, page=32),
        # A large cache's scattered pages brought together: bytes.
        dict(name="copy_compact", kind="copy", n=12000, pages=30000, hkv=8, d=128, bits=4, page=32),
        # Eight answers to one short prompt: latency.
        dict(name="shared_short_8", kind="shared", b=8, groups=1, shared=1000, kv=1300, q=1, hq=32, hkv=8, d=128, bits=8, page=16),
        # 64 requests behind one long document: its keys once, 256 query rows to a key head.
        dict(name="shared_long_64", kind="shared", b=64, groups=1, shared=32768, kv=33500, q=1, hq=32, hkv=8, d=128, bits=8, page=64),
        # Five documents, several requests to each, two tokens at a time, narrow heads, prefixes that end inside pages.
        dict(name="shared_groups", kind="shared", b=27, groups=5, shared=4999, kv=7001, q=2, hq=28, hkv=4, d=64, bits=4, page=16),
        # One short prompt: latency, few compute units.
        dict(name="prompt_short_333", kind="prompt", b=1, n=333, hq=32, hkv=8, d=128, causal=True, window=0),
        # Long prompts, four query heads to a key head: matrix operations.
        dict(name="prompt_long_8192", kind="prompt", b=2, n=8192, hq=32, hkv=8, d=128, causal=True, window=0),
        # Many ragged prompts packed one behind the other, narrow heads, a key head per query head, a sliding window.
        dict(name="prompt_packed_window", kind="prompt", b=21, n=2001, hq=12, hkv=12, d=64, causal=True, window=777),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case of the same ranges: 1 to 16384 tokens, 1 to 64 sequences of 1 to 33500 tokens of context, prompts of 1
    to 8192 tokens, all head layouts, types and options."""
    kind = rng.choice(["rotary", "rotary", "into", "into", "copy", "copy", "shared", "shared", "shared", "prompt", "prompt", "prompt", "prompt"])
    d = rng.choice([64, 128, 128, 128, 96, 80, 256])
    rot = rng.choice([d, d, 16 * (d // 32), 16 * max(1, d // 64)])
    hq, hkv = rng.choice([(32, 32), (32, 8), (64, 8), (28, 4), (16, 1), (12, 12), (8, 4)])
    factor = rng.choice([1.0, 1.0, 2.0, 8.0, 32.0])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "rotary":
        heads = rng.choice([hq, hkv, hq + hkv])
        t = min(int(_log(rng, 1, 16385)), int(8.3e7 / (heads * d)))
        rot = rng.choice([rot, 2 * rng.randint(1, d // 2)])
        return dict(kind=kind, t=t, heads=heads, d=d, rot=rot, interleaved=rng.choice([True, False]), dtype=dtype, factor=factor,
                    far=int(_log(rng, 1000, 1000001)))
    bits = rng.choice([8, 8, 4])
    page = rng.choice([1, 8, 16, 32, 64, 256])
    if kind == "into":
        b = int(_log(rng, 1, 65))
        hq, hkv = rng.choice([(hq, hkv), (4, 4), (4, 1)])
        most = 6e8 / ((2 * hq + 4 * hkv) * d * _BYTES[dtype])   # tokens
        b = max(1, min(b, int(most)))
        kv = max(1, min(int(_log(rng, 1, 8193)), int(most / b)))
        return dict(kind=kind, b=b, kv=kv, new=rng.choice([1, 1, kv, max(1, kv // 3)]), hq=hq, hkv=hkv, d=d, rot=rot,
                    interleaved=rng.choice([True, False]), bits=bits, page=page, dtype=dtype, factor=factor)
    if kind == "copy":
        per = 2 * hkv * page * (d * bits // 8 + 5)
        n = min(int(_log(rng, 1, 20001)), max(1, int(4e8 / per)))
        return dict(kind=kind, n=n, pages=2 * n + int(_log(rng, 1, 1 + min(n, 1000) + 100)), hkv=hkv, d=d, bits=bits, page=page)
    if kind == "shared":
        b = int(_log(rng, 1, 65))
        shared = int(_log(rng, 1, 32769))
        kv = shared + int(_log(rng, 1, 2001))
        b = max(1, min(b, int(5.0e8 / (hkv * d * kv))))
        q = rng.choice([1, 1, 1, max(1, 16 * hkv // hq), rng.randint(1, 3)])
        return dict(kind=kind, b=b, groups=rng.randint(1, max(1, b // 3)), shared=shared, kv=kv, q=min(q, kv - shared), hq=hq, hkv=hkv, d=d, bits=bits, page=page)
    causal = rng.choice([True, True, True, False])
    n = int(_log(rng, 1, 8193))
    most = (2.6e9 if causal else 1.3e9) / (hq * max(1.0, d / 128))   # pairs of tokens
    n = min(n, int(math.sqrt(most)))
    b = max(1, min(int(_log(rng, 1, 33)), int(most / (n * n)), int(8e8 / (4 * (hq + hkv) * d * n))))
    return dict(kind=kind, b=b, n=n, hq=hq, hkv=hkv, d=d, causal=causal, window=int(_log(rng, 16, 4097)) if rng.random() < 0.25 else 0)


def _part(i):
    """Between a fifth and all: sequences differ, the first has all that the case says."""
    return 1.0 - 0.8 * ((i * 0.6180339887) % 1.0)


def _lengths(case):
    """Tokens that every sequence holds, and how many of them are new."""
    if case["kind"] == "prompt":
        n = [max(1, int(round(case["n"] * _part(i)))) for i in range(case["b"])]
        return n, n
    kv, new = [], []
    for i in range(case["b"]):
        if case["kind"] == "shared":
            common, q = _prefixes(case)[_group(case, i)], case["q"]
            k = common + max(q, int(round((case["kv"] - case["shared"]) * _part(i))))
        else:
            k = max(1, int(round(case["kv"] * _part(i))))
            q = case["new"] if i == 0 or case["new"] == 1 else max(1, int(round(case["new"] * _part(i))))
        kv.append(k)
        new.append(min(k, q))
    return kv, new


def _group(case, i):
    """Sequences of a group lie side by side."""
    return i * case["groups"] // case["b"]


def _prefixes(case):
    return [max(1, int(round(case["shared"] * _part(j)))) for j in range(case["groups"])]


def _visible(case):
    """Pairs of a query and a key that it sees, of one head."""
    causal, window = case.get("causal", True), case.get("window", 0)
    total = 0
    for k, q in zip(*_lengths(case)):
        for pos in (range(k - q, k) if causal or window else ()):
            hi = pos + 1 if causal else k
            total += hi - (max(0, pos - window + 1) if window else 0)
        if not causal and not window:
            total += q * k
    return total


def _cache_bytes(tokens, case):
    return 2 * tokens * case["hkv"] * (case["d"] * case["bits"] // 8 + 5)


def work(case):
    k, d = case["kind"], case["d"]
    if k == "rotary":
        e = case["t"] * case["heads"]
        return {"bytes": 2 * e * d * _BYTES[case["dtype"]] + 4 * case["t"] + 4 * case["rot"], "flops": 3 * e * case["rot"]}
    if k == "copy":
        return {"bytes": 2 * _cache_bytes(case["n"] * case["page"], case) + 8 * case["n"], "flops": 0}
    kv, new = _lengths(case)
    if k == "into":
        b, written, read = _BYTES[case["dtype"]], sum(new), sum(kv)
        nbytes = written * (2 * case["hq"] + 2 * case["hkv"]) * d * b + 8 * written + _cache_bytes(written + read, case) + 2 * read * case["hkv"] * d * b
        return {"bytes": nbytes, "flops": 3 * written * (case["hq"] + case["hkv"]) * case["rot"] + 6 * written * 2 * case["hkv"] * d}
    if k == "shared":
        common = _prefixes(case)
        distinct = sum(common) + sum(n - common[_group(case, i)] for i, n in enumerate(kv))
        return {"bytes": 4 * sum(new) * case["hq"] * d + _cache_bytes(distinct, case), "flops": 4 * d * case["hq"] * _visible(case)}
    return {"bytes": 2 * sum(kv) * d * (2 * case["hq"] + 2 * case["hkv"]), "flops": 4 * d * case["hq"] * _visible(case)}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + tag) & 0x7FFFFFFFFFFF)
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=F32)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _frequencies(case):
    """Of the pairs of channels: powers of 10000, those that turn less than once in 8192 tokens slowed by the factor, those that turn
    more than four times as they are, and in between in proportion."""
    f = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=F64, device="cuda") / case["rot"])
    kept = ((f * (8192 / (2 * math.pi)) - 1.0) / 3.0).clamp(0.0, 1.0)
    return f * (kept + (1.0 - kept) / case["factor"])


def _magnitude(case):
    return 1.0 + 0.1 * math.log(case["factor"])


def _filled(case, pages, g):
    """A cache full of quantized normal keys (channels of different scales) and values."""
    hkv, page, d, bits = case["hkv"], case["page"], case["d"], case["bits"]
    codes = torch.empty((2, pages, hkv, page, d * bits // 8), dtype=torch.uint8, device="cuda")
    scales = torch.empty((2, pages, hkv, page), dtype=F32, device="cuda")
    zeros = torch.empty((2, pages, hkv, page), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (hkv * page * d))
    spread = torch.exp(0.4 * _randn((hkv, 1, d), g))
    for which in range(2):
        for a in range(0, pages, step):
            x = _randn((min(step, pages - a), hkv, page, d), g)
            x = (x * spread if which == 0 else x).bfloat16().float()
            c, s, z = _grid(x, bits)
            codes[which, a:a + step], scales[which, a:a + step], zeros[which, a:a + step] = _pack(c, bits), s, z
    return codes, scales, zeros


def _tables(case, kv, g):
    """A page table over pages in random order, a few of which belong to no sequence; sequences of a group have the pages that their
    prefix fills in common, and each a copy of the one in which it ends."""
    page = case["page"]
    used = [-(-n // page) for n in kv]
    owned, common = [], []
    for i, u in enumerate(used):
        full = 0
        if case["kind"] == "shared" and i > 0 and _group(case, i) == _group(case, i - 1):
            full = _prefixes(case)[_group(case, i)] // page
        common.append(full)
        owned.append(u - full)
    pages = sum(owned) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((len(kv), max(used)), dtype=torch.int32, device="cuda")
    at = 0
    for i, u in enumerate(used):
        if common[i]:
            table[i, :common[i]] = table[i - 1, :common[i]]
        table[i, common[i]:u] = order[at:at + owned[i]]
        at += owned[i]
    return table, pages


def prepare(case, seed):
    k, d = case["kind"], case["d"]
    s = dict(case)
    g = _gen(seed, 2)
    if k == "rotary":
        dt = _DTYPES[case["dtype"]]
        # the heads lie in a projection's output, whose last heads' values stay as they are
        s["X"] = _randn((case["t"], case["heads"] + 2, d), g).to(dt)[:, :case["heads"]]
        s["Y"] = torch.empty((case["t"], case["heads"], d), dtype=dt, device="cuda")
        s["positions"] = torch.randint(0, case["far"], (case["t"],), generator=g, device="cuda", dtype=torch.int32)
        s["freq"], s["scale"] = _frequencies(case), _magnitude(case)
        return s
    if k == "copy":
        s["codes"], s["scales"], s["zeros"] = _filled(case, case["pages"], g)
        order = torch.randperm(case["pages"], generator=g, device="cuda").to(torch.int32)
        s["source"], s["target"] = order[:case["n"]].contiguous(), order[case["n"]:2 * case["n"]].contiguous()
        return s
    kv, new = _lengths(case)
    if k == "prompt":
        t = sum(kv)
        # one projection's output: queries, keys and values side by side
        qkv = _randn((t, case["hq"] + 2 * case["hkv"], d), g).bfloat16()
        s["Q"], s["K"], s["V"] = qkv.split([case["hq"], case["hkv"], case["hkv"]], dim=1)
        s["cu"], s["max_n"] = _ints(_starts(kv)), max(kv)
        s["O"] = torch.empty((t, case["hq"], d), dtype=torch.bfloat16, device="cuda")
        s["softmax_scale"] = 1.0 / math.sqrt(d)
        return s
    s["table"], s["pages"] = _tables(case, kv, g)
    s["codes"], s["scales"], s["zeros"] = _filled(case, s["pages"], g)
    s["kv_lens"], s["cu_q"] = _ints(kv), _ints(_starts(new))
    s["max_kv"], s["max_q"] = max(kv), max(new)
    t = sum(new)
    if k == "shared":
        for i in range(1, case["b"]):   # the page in which a prefix ends: each sequence's own copy of its beginning
            j, page = _group(case, i), case["page"]
            n = _prefixes(case)[j]
            if j == _group(case, i - 1) and n % page:
                src, dst = s["table"][i - 1, n // page], s["table"][i, n // page]
                for c in (s["codes"], s["scales"], s["zeros"]):
                    c[:, dst, :, :n % page] = c[:, src, :, :n % page]
        first = [next(i for i in range(case["b"]) if _group(case, i) == j) for j in range(case["groups"])]
        s["cu_groups"], s["shared_lens"], s["max_shared"] = _ints(first + [case["b"]]), _ints(_prefixes(case)), max(_prefixes(case))
        s["Q"] = _randn((t, case["hq"], d), g).bfloat16()
        s["O"] = torch.empty_like(s["Q"])
        s["softmax_scale"] = 1.0 / math.sqrt(d)
        return s
    dt = _DTYPES[case["dtype"]]
    seq = torch.repeat_interleave(torch.arange(case["b"], device="cuda"), _ints(new).long())
    place = torch.arange(t, device="cuda") - s["cu_q"][seq] + (s["kv_lens"] - _ints(new))[seq]
    s["positions"] = place.to(torch.int32)
    s["slots"] = (s["table"][seq, place // case["page"]] * case["page"] + place % case["page"]).to(torch.int32)
    qkv = _randn((t, case["hq"] + 2 * case["hkv"], d), g)
    qkv[:, case["hq"]:case["hq"] + case["hkv"]] *= torch.exp(0.4 * _randn((case["hkv"], d), g))
    s["Q"], s["K"], s["V"] = qkv.to(dt).split([case["hq"], case["hkv"], case["hkv"]], dim=1)
    s["Q_out"] = torch.empty((t, case["hq"], d), dtype=dt, device="cuda")
    s["freq"], s["scale"] = _frequencies(case), _magnitude(case)
    s["cu_kv"] = _ints(_starts(kv))
    s["K_back"] = torch.empty((sum(kv), case["hkv"], d), dtype=dt, device="cuda")
    s["V_back"] = torch.empty_like(s["K_back"])
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _PLAIN[s["kind"]](s)


def _run_own(s):
    import paper_2601_19675_amd as ptq
    k = s["kind"]
    if k == "rotary":
        ptq.ptq_rotary(s["X"], s["positions"], s["freq"], s["Y"], scale=s["scale"], interleaved=s["interleaved"])
        return {"Y": s["Y"]}
    if k == "into":
        ptq.ptq_rotary_kv_cache_write(s["Q"], s["K"], s["V"], s["positions"], s["freq"], s["slots"], s["bits"], s["codes"], s["scales"], s["zeros"],
                                      s["Q_out"], scale=s["scale"], interleaved=s["interleaved"])
        ptq.ptq_kv_cache_read(s["codes"], s["scales"], s["zeros"], s["bits"], s["table"], s["cu_kv"], s["max_kv"], s["K_back"], s["V_back"])
        return {"Q": s["Q_out"], "K": s["K_back"], "V": s["V_back"]}
    if k == "copy":
        ptq.ptq_kv_cache_copy_pages(s["codes"], s["scales"], s["zeros"], s["source"], s["codes"], s["scales"], s["zeros"], s["target"])
        return {"codes": s["codes"], "scales": s["scales"], "zeros": s["zeros"]}
    if k == "shared":
        if "ws" not in s:   # a program keeps its workspace
            s["ws"] = torch.empty(max(256, ptq.ptq_workspace_bytes(ptq.OP_SHARED_ATTENTION, s["hq"], s["d"], s["Q"].shape[0], s["max_kv"])),
                                  dtype=torch.uint8, device="cuda")
        ptq.ptq_paged_attention_shared(s["Q"], s["cu_q"], s["max_q"], s["codes"], s["scales"], s["zeros"], s["bits"], s["table"], s["kv_lens"],
                                       s["max_kv"], s["cu_groups"], s["shared_lens"], s["max_shared"], s["softmax_scale"], s["O"], ws=s["ws"])
        return {"O": s["O"]}
    ptq.ptq_prompt_attention(s["Q"], s["K"], s["V"], s["cu"], s["max_n"], s["softmax_scale"], s["O"], causal=s["causal"], window=s["window"])
    return {"O": s["O"]}


# ---------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------
def _turned(x, s):
    """x [tokens, heads, width] with its first channels turned, pair by pair, rounded once to its type."""
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = (s["scale"] * torch.cos(angle))[:, None], (s["scale"] * torch.sin(angle))[:, None]
    half = s["freq"].numel()
    v = x.double()
    a, b = (v[..., 0:2 * half:2], v[..., 1:2 * half:2]) if s["interleaved"] else (v[..., :half], v[..., half:2 * half])
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((a, b), dim=-1).flatten(-2) if s["interleaved"] else torch.cat((a, b), dim=-1)
    return torch.cat((y, v[..., 2 * half:]), dim=-1).to(x.dtype)


def _rotary(s):
    return {"Y": _turned(s["X"], s)}


def _copy(s):
    source, target = s["source"].long(), s["target"].long()
    for c in (s["codes"], s["scales"], s["zeros"]):
        c[:, target] = c[:, source]
    return {"codes": s["codes"], "scales": s["scales"], "zeros": s["zeros"]}


def _grid(x, bits):
    """Codes, scale and zero of every row: the asymmetric grid that holds the row's values and 0."""
    top = 2 ** bits - 1
    x = x.double()
    lo, hi = x.amin(dim=-1).clamp(max=0.0), x.amax(dim=-1).clamp(min=0.0)
    flat = lo == hi
    lo, hi = torch.where(flat, -1.0, lo), torch.where(flat, 1.0, hi)
    scale = ((hi - lo) / top).float()
    zero = torch.round(-lo / scale.double())
    code = (torch.round(x / scale.double()[..., None]) + zero[..., None]).clamp(0, top)
    return code.to(torch.uint8), scale, zero.to(torch.uint8)


def _pack(code, bits):
    if bits == 8:
        return code
    c = code.reshape(code.shape[:-1] + (-1, 4, 2))                 # words, i, even / odd
    c = c.transpose(-1, -2).reshape(c.shape[:-2] + (4, 2))         # bytes of a word, low / high half
    return (c[..., 0] | (c[..., 1] << 4)).reshape(code.shape[:-1] + (-1,))


def _unpack(packed, bits):
    if bits == 8:
        return packed
    c = torch.stack((packed & 15, packed >> 4), dim=-1).reshape(packed.shape[:-1] + (-1, 2, 4))
    return c.transpose(-1, -2).reshape(packed.shape[:-1] + (-1,))


def _gathered(s, which, page, offset):
    """Float32 keys (0) or values (1) of cache places, which page and where in it: [.., heads, width]."""
    code = _unpack(s["codes"][which][page, :, offset], s["bits"]).float()
    return s["scales"][which][page, :, offset][..., None] * (code - s["zeros"][which][page, :, offset][..., None].float())


def _into(s):
    page, offset = (s["slots"] // s["page"]).long(), (s["slots"] % s["page"]).long()
    for which, x in ((0, _turned(s["K"], s)), (1, s["V"])):
        code, scale, zero = _grid(x, s["bits"])
        s["codes"][which][page, :, offset] = _pack(code, s["bits"])
        s["scales"][which][page, :, offset] = scale
        s["zeros"][which][page, :, offset] = zero
    rows = torch.arange(s["K_back"].shape[0], device="cuda")
    seq = torch.searchsorted(s["cu_kv"][1:].contiguous(), rows.to(torch.int32), right=True)
    place = rows - s["cu_kv"][seq]
    page = s["table"][seq, place // s["page"]].long()
    return {"Q": _turned(s["Q"], s), "K": _gathered(s, 0, page, place % s["page"]).to(s["K"].dtype),
            "V": _gathered(s, 1, page, place % s["page"]).to(s["V"].dtype)}


def _softmax_product(q, K, V, seen, scale):
    """q [b, heads, rows, width] against K [b, heads, width, keys], V [b, heads, keys, width] where seen [b, 1, rows, keys]."""
    scores = (q @ K).mul_(scale).masked_fill_(~seen, -math.inf)
    p = scores.sub_(scores.amax(dim=-1, keepdim=True).clamp_(min=-3e38)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    return torch.where(total > 0, 1.0 / total, 0.0) * (p @ V)


def _shared(s):
    """Softmax attention of every sequence's last tokens, padded to the longest, in float32."""
    b, lq, lk, hq, hkv, d = s["b"], s["max_q"], s["max_kv"], s["hq"], s["hkv"], s["d"]
    t, group = s["Q"].shape[0], hq // hkv
    new = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    i, j = torch.arange(lq, device="cuda"), torch.arange(lk, device="cuda")
    row = (s["cu_q"][:-1, None] + i).clamp(max=t - 1).long()
    q = s["Q"][row].float().view(b, lq, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, d)
    there = j < s["kv_lens"][:, None]
    page = torch.where(there, s["table"][:, j // s["page"]], 0).long()
    offset = (j % s["page"]).expand(b, lk)
    seen = there[:, None] & (j <= ((s["kv_lens"].long() - new)[:, None] + i)[:, :, None])
    seen = seen[:, None].expand(b, group, lq, lk).reshape(b, 1, group * lq, lk)
    K = _gathered(s, 0, page, offset).permute(0, 2, 3, 1).contiguous()
    V = torch.where(there[:, :, None, None], _gathered(s, 1, page, offset), 0.0).transpose(1, 2).contiguous()
    O = _softmax_product(q, K, V, seen, s["softmax_scale"]).view(b, hq, lq, d)
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), new, output_size=t)
    return {"O": O[seq, :, torch.arange(t, device="cuda") - s["cu_q"][seq]].to(s["Q"].dtype)}


def _prompt(s):
    """Softmax attention of every prompt, padded to the longest, in float32."""
    b, n, hq, hkv, d = s["b"], s["max_n"], s["hq"], s["hkv"], s["d"]
    t, group = s["Q"].shape[0], hq // hkv
    lens = (s["cu"][1:] - s["cu"][:-1]).long()
    i = torch.arange(n, device="cuda")
    row = (s["cu"][:-1, None] + i).clamp(max=t - 1).long()
    q = s["Q"][row].float().view(b, n, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, group * n, d)
    there = i < lens[:, None]
    K = s["K"][row].float().permute(0, 2, 3, 1).contiguous()
    V = torch.where(there[:, :, None, None], s["V"][row].float(), 0.0).transpose(1, 2).contiguous()
    seen = there[:, None, :].expand(b, n, n)
    if s["causal"]:
        seen = seen & (i <= i[:, None])
    if s["window"]:
        seen = seen & (i > i[:, None] - s["window"])
    seen = seen[:, None].expand(b, group, n, n).reshape(b, 1, group * n, n)
    O = _softmax_product(q, K, V, seen, s["softmax_scale"]).view(b, hq, n, d)
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), lens, output_size=t)
    return {"O": O[seq, :, torch.arange(t, device="cuda") - s["cu"][seq]].to(s["Q"].dtype)}


_PLAIN = {"rotary": _rotary, "into": _into, "copy": _copy, "shared": _shared, "prompt": _prompt}


# ---------------------------------------------------------------------------------------------
# the definitions in float64
# ---------------------------------------------------------------------------------------------
def _rotated(x, s, case):
    """Pairs of channels as complex numbers, multiplied by scale e^(i angle)."""
    z = torch.polar(torch.full_like(s["freq"], s["scale"]).expand(x.shape[0], -1).contiguous(), torch.outer(s["positions"].to(F64), s["freq"]))
    out, n = x.to(F64).clone(), case["rot"]
    first, second = (slice(0, n, 2), slice(1, n, 2)) if case["interleaved"] else (slice(0, n // 2), slice(n // 2, n))
    pair = torch.complex(out[..., first], out[..., second]) * z[:, None, :]
    out[..., first], out[..., second] = pair.real, pair.imag
    return out


def _row_values(x, bits):
    """What a row of the cache stands for once x has been stored in it (float64)."""
    levels = float((1 << bits) - 1)
    x = x.to(F64)
    low = torch.minimum(x.min(dim=-1, keepdim=True).values, torch.zeros((), dtype=F64, device="cuda"))
    high = torch.maximum(x.max(dim=-1, keepdim=True).values, torch.zeros((), dtype=F64, device="cuda"))
    empty = high - low == 0
    low, high = low.masked_fill(empty, -1.0), high.masked_fill(empty, 1.0)
    step = ((high - low) / levels).to(F32).to(F64)
    origin = (-low / step).round()
    return step * (((x / step).round() + origin).clamp(0.0, levels) - origin)


def _held(s, which, i, length):
    """Keys or values that the cache holds for sequence i, place by place (float64, [length, heads, width])."""
    pages = s["table"][i, : -(-length // s["page"])].long()
    code = s["codes"][which, pages].to(torch.int32)
    if s["bits"] == 4:
        word = sum(code[..., byte::4].long() << (8 * byte) for byte in range(4))
        code = torch.stack([(word >> (4 * (e // 2) + 16 * (e % 2))) & 15 for e in range(8)], dim=-1).flatten(-2)
    x = s["scales"][which, pages].to(F64)[..., None] * (code.to(F64) - s["zeros"][which, pages].to(F64)[..., None])
    return x.transpose(1, 2).flatten(0, 1)[:length]


def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "rotary":
        return {"Y": _rotated(s["X"], s, case)}
    if k == "copy":
        out = {"codes": s["codes"].clone(), "scales": s["scales"].clone(), "zeros": s["zeros"].clone()}
        for name in out:
            out[name].index_copy_(1, s["target"].long(), s[name].index_select(1, s["source"].long()))
        return dict(out, scales=out["scales"].to(F64))
    kv, new = _lengths(case)
    if k == "into":
        # a turned key is rounded to its type before it is quantized
        K = _rotated(s["K"], s, case).to(s["K"].dtype)
        back, at = {"K": [], "V": []}, 0
        for i, (c, q) in enumerate(zip(kv, new)):
            for which, name, x in ((0, "K", K), (1, "V", s["V"])):
                back[name] += [_held(s, which, i, c - q), _row_values(x[at:at + q], case["bits"])]
            at += q
        return dict({name: torch.cat(parts) for name, parts in back.items()}, Q=_rotated(s["Q"], s, case))
    group, at, out = case["hq"] // case["hkv"], 0, torch.zeros(s["Q"].shape, dtype=F64, device="cuda")
    causal, window = case.get("causal", True), case.get("window", 0)
    for i, (c, q) in enumerate(zip(kv, new)):
        K, V = (s["K"][at:at + c].to(F64), s["V"][at:at + c].to(F64)) if k == "prompt" else (_held(s, 0, i, c), _held(s, 1, i, c))
        keys, places = torch.arange(c, device="cuda")[None, :], torch.arange(c - q, c, device="cuda")[:, None]
        hidden = torch.zeros((q, c), dtype=torch.bool, device="cuda")
        if causal:
            hidden |= keys > places
        if window:
            hidden |= keys <= places - window
        for h in range(case["hq"]):
            logits = torch.mm(s["Q"][at:at + q, h].to(F64), K[:, h // group].t()) * s["softmax_scale"]
            out[at:at + q, h] = torch.mm(torch.softmax(logits.masked_fill(hidden, -math.inf), dim=-1), V[:, h // group])
        at += q
    return {"O": out}
