"""Performance cases of the attention operators: rotary positions with several axes, attention with a sliding window
and first tokens that stay visible, and the 8-bit cache of keys and values (filling it, attention over it).

A case says which operator is called (`op`) and with what sizes; `prepare` makes what a program holds before the call,
`run` makes the call once: with `own` through this library's entry points, else in plain torch, in 32 bits and rounded
once at the end.  `exact` is the operator's definition in 64 bits, `work` what a call cannot do without.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
PAGE = 64                 # tokens in a page of the 8-bit cache, which share a scale for each head
ALL = 2147483647          # a window without an end


def _rope(type, T, Hq, Hk, D, sections, pairing):
    s = tuple(sections) + (0,) * (4 - len(sections))
    return {"op": "rope", "type": type, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "axes": len(sections),
            "s0": s[0], "s1": s[1], "s2": s[2], "s3": s[3], "pairing": pairing}


def _attn(type, B, Lq, Lk, Hq, Hk, D, left, right, sinks, mix):
    # mix 0: B sequences of Lq queries and Lk keys; else lengths up to those, by this number
    return {"op": "attn", "type": type, "B": B, "Lq": Lq, "Lk": Lk, "Hq": Hq, "Hk": Hk, "D": D, "left": left,
            "right": right, "sinks": sinks, "mix": mix}


def _append(type, B, new, have, Hk, D, mix):
    # B sequences that hold `have` tokens get `new` more each (mix: up to those)
    return {"op": "append", "type": type, "B": B, "new": new, "have": have, "Hk": Hk, "D": D, "mix": mix}


def _kv8(type, B, Lq, L, Hq, Hk, D, left, sinks, mix):
    # B sequences of L cached tokens (mix: up to that), the last Lq of which ask
    return {"op": "kv8", "type": type, "B": B, "Lq": Lq, "L": L, "Hq": Hq, "Hk": Hk, "D": D, "left": left,
            "sinks": sinks, "mix": mix}


def listed():
    return [
        # one step of serving: a new token of each of eight volumes gets its positions
        {"name": "rope_step_8", **_rope("bf16", 8, 16, 4, 128, (16, 24, 24), "halves")},
        # the voxels of a whole 32^3 feature map
        {"name": "rope_volume_32", **_rope("bf16", 32768, 16, 4, 128, (16, 24, 24), "halves")},
        # a 14^3 map as the layers leave it (fp32), narrow heads, a part of each head without positions
        {"name": "rope_odd_14", **_rope("f32", 2744, 5, 5, 40, (5, 6, 6), "neighbours")},
        # short sequences of very different lengths, some of them empty, in one call
        {"name": "attn_ragged", **_attn("f16", 9, 300, 333, 8, 8, 64, 100, 0, 4, 5)},
        # a 14^3 map in fp32, each voxel sees the slabs before and behind it
        {"name": "attn_slabs_f32", **_attn("f32", 1, 2744, 2744, 5, 5, 40, 392, 392, 0, 0)},
        # a whole volume of 16 x 32 x 32 voxels, the last four slabs and the first tokens visible: the largest
        {"name": "attn_volume", **_attn("bf16", 1, 16384, 16384, 16, 4, 128, 4095, 0, 16, 0)},
        # one new token of each of eight sequences against all keys before it, unquantised
        {"name": "attn_token_8k", **_attn("bf16", 8, 1, 8192, 16, 4, 128, ALL, 0, 0, 0)},
        # one step of serving: a token of each of 64 sequences goes into the cache
        {"name": "append_step_64", **_append("bf16", 64, 1, 5000, 8, 128, 3)},
        # two prompts go into the cache
        {"name": "append_prompt", **_append("bf16", 2, 16384, 40, 8, 128, 0)},
        # a single short sequence: the smallest step
        {"name": "kv8_step_777", **_kv8("f16", 1, 1, 777, 16, 4, 64, ALL, 0, 0)},
        # a serving batch of ragged lengths with a window and sinks
        {"name": "kv8_window_64", **_kv8("bf16", 64, 1, 32768, 16, 4, 128, 4095, 64, 7)},
        # long sequences, everything visible: the pools pass 32-bit offsets
        {"name": "kv8_long_131072", **_kv8("bf16", 32, 1, 131072, 32, 8, 128, ALL, 0, 0)},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more call of the ranges that the listed ones span, never dearer than the largest of them."""
    while True:
        op, type = rng.choice(("rope", "attn", "attn", "append", "kv8", "kv8")), rng.choice(("f32", "bf16", "bf16", "f16"))
        Hk = rng.choice((1, 2, 3, 4, 5, 8, 16))
        G = rng.choice((1, 1, 2, 3, 4, 5, 8))
        D = 8 * rng.randint(2, 16) if rng.random() < 0.5 else rng.choice((64, 128))
        mix = rng.choice((0, rng.randint(1, 99)))
        if Hk * G > 48:
            continue
        if op == "rope":
            A = rng.choice((1, 2, 3, 3, 3, 4))
            R = D // 2 if rng.random() < 0.7 else rng.randint(A, D // 2)
            cuts = sorted(rng.sample(range(1, R), A - 1)) if R > A else list(range(1, A))
            s = [b - a for a, b in zip([0] + cuts, cuts + [max(R, A)])]
            c = _rope(type, _log(rng, 1, 32768), Hk * G, Hk, D, s, rng.choice(("halves", "neighbours")))
            if work(c)["bytes"] > 3.3e8:
                continue
        elif op == "attn":
            B = _log(rng, 1, 32)
            if rng.random() < 0.25:
                Lq, Lk = rng.randint(1, 8), _log(rng, 1, 16384)
            else:
                Lk = _log(rng, 1, 16384)
                Lq = Lk if rng.random() < 0.6 else _log(rng, 1, Lk)
            left = ALL if rng.random() < 0.2 else _log(rng, 1, 8192) - 1
            right = rng.choice((0, 0, 0, left, ALL))
            c = _attn(type, B, Lq, Lk, Hk * G, Hk, D, left, right, rng.choice((0, 1, 4, 16, 100)), mix)
            dense = 4.0 * B * Hk * G * Lq * Lk * D
            if B * Hk * G * Lq * Lk > 2.0e9 or dense > (1e11 if type == "f32" else 4.8e11):
                continue
        elif op == "append":
            if rng.random() < 0.4:
                B, new = _log(rng, 1, 128), rng.randint(1, 4)
            else:
                B, new = _log(rng, 1, 16), _log(rng, 1, 16384)
            c = _append(type, B, new, _log(rng, 1, 8192) - 1, Hk, D, mix)
            if B * (c["new"] + c["have"]) * Hk * D > 1.0e8:
                continue
        else:
            left = ALL if rng.random() < 0.5 else _log(rng, 1, 16384) - 1
            c = _kv8(type, _log(rng, 1, 128), rng.choice((1, 1, 1, 2, 3, 4, 7)), _log(rng, 1, 131072), Hk * G, Hk, D, left,
                     rng.choice((0, 0, 4, 64, 100)), mix)
            if c["B"] * c["L"] * Hk * D > 2.0e9 or c["B"] * c["L"] * Hk * G * c["Lq"] > 1.0e9:
                continue
        if 3072 not in (*c.values(), Hk * D, Hk * G * D):
            return c


# ---- sizes that follow from a case ---------------------------------------------------------------------------------

def _lengths(c):
    """Of each sequence of the case: (queries, keys), (new, held) or cached tokens."""
    r, B = random.Random(c["mix"]), c["B"]
    if c["op"] == "attn":
        if not c["mix"]:
            return [(c["Lq"], c["Lk"])] * B
        got = [(r.randint(0, c["Lq"]), r.randint(0, c["Lk"])) for _ in range(B)]   # fewer keys than queries: rows see none
        return [(q, k if r.random() < 0.3 else max(q, k)) for q, k in got[:-1]] + [(c["Lq"], c["Lk"])]
    if c["op"] == "append":
        if not c["mix"]:
            return [(c["new"], c["have"])] * B
        return [(r.randint(0, c["new"]) if c["new"] > 1 else 1, r.randint(0, c["have"])) for _ in range(B - 1)] + [(c["new"], c["have"])]
    if not c["mix"]:
        return [c["L"]] * B
    return [r.randint(0, c["L"]) for _ in range(B - 1)] + [c["L"]]


def _pages(n):
    return -(-n // PAGE)


def _seen(p, n, left, right, sinks):
    """How many of n keys a row at position p sees."""
    hi = min(n - 1, p + right)
    lo = max(0, p - left)
    return max(0, hi - lo + 1) + max(0, min(sinks, lo, hi + 1))


def _span(lq, lk, left, right, sinks):
    """How many of lk keys any of lq rows, the last of which stands at lk - 1, sees."""
    if not lq:
        return 0
    first = min(lk, max(0, lk - lq - left))
    return min(lk, lk + right) - first + min(sinks, first)


def work(case):
    c, b = case, SIZE[case["type"]]
    if c["op"] == "rope":
        R = c["s0"] + c["s1"] + c["s2"] + c["s3"]
        values = c["T"] * (c["Hq"] + c["Hk"]) * c["D"]
        return {"bytes": 2 * b * values + 4 * c["T"] * c["axes"] + 4 * R, "flops": 3 * values}
    n = _lengths(c)
    if c["op"] == "attn":
        # (arithmetic series would do; a sum over rows of a few ten thousand is quick enough)
        seen = 0
        for (lq, lk), times in {x: n.count(x) for x in n}.items():
            seen += times * sum(_seen(lk - lq + i, lk, c["left"], c["right"], c["sinks"]) for i in range(lq))
        nq, nk = sum(q for q, _ in n), sum(_span(q, k, c["left"], c["right"], c["sinks"]) for q, k in n)
        return {"bytes": b * c["D"] * (2 * nq * c["Hq"] + 2 * nk * c["Hk"]), "flops": 4.0 * seen * c["Hq"] * c["D"]}
    if c["op"] == "append":
        new = sum(a for a, _ in n)
        return {"bytes": 2 * new * c["Hk"] * c["D"] * (b + 1), "flops": 4.0 * new * c["Hk"] * c["D"]}
    keys = sum(_span(min(c["Lq"], l), l, c["left"], 0, c["sinks"]) for l in n)
    return {"bytes": 2 * keys * c["Hk"] * c["D"] + 2 * b * c["B"] * c["Lq"] * c["Hq"] * c["D"],
            "flops": 4.0 * keys * c["Lq"] * c["Hq"] * c["D"]}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _starts(v):
    t = [0]
    for x in v:
        t.append(t[-1] + x)
    return t


def _cache(c, g, lens, spare):
    """Pools of 8-bit pages, their scales, and a table of pages in no order; slots past a sequence's end hold zeros."""
    Hk, D, B = c["Hk"], c["D"], c["B"]
    width = max(1, max(_pages(x) for x in lens)) + spare
    pages = B * width
    kc = torch.empty((pages, Hk, PAGE, D), dtype=torch.uint8, device=DEVICE)
    vc = torch.empty((pages, Hk, D, PAGE), dtype=torch.uint8, device=DEVICE)
    step = max(1, (1 << 28) // (Hk * PAGE * D))
    for pool in (kc, vc):
        for at in range(0, pages, step):
            part = pool[at:at + step]
            x = torch.randn(part.shape, dtype=torch.bfloat16, device=DEVICE, generator=g).mul_(96).clamp_(-448, 448)
            part.copy_(x.to(torch.float8_e4m3fn).view(torch.uint8))
    scales = torch.exp2(torch.randint(-8, -5, (pages, Hk, 2), device=DEVICE, generator=g).float())
    table = torch.randperm(pages, device=DEVICE, generator=g).to(torch.int32).view(B, width)
    return kc, vc, scales, table


def _axis_of_pair(sections):
    return sum(([a] * n for a, n in enumerate(sections)), [])


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = TYPES[c["type"]]

    def normal(*shape):
        return torch.randn(shape, device=DEVICE, generator=g).to(dt)

    if c["op"] == "rope":
        s = [c["s%d" % a] for a in range(c["axes"])]
        edge = min(1024, 4 * max(1, round(c["T"] ** (1.0 / c["axes"]))))      # images have edges up to 1024
        pos = torch.randint(0, edge, (c["T"], c["axes"]), device=DEVICE, generator=g, dtype=torch.int32)
        freq = torch.cat([10000.0 ** (-torch.arange(n, device=DEVICE, dtype=torch.float32) / n) for n in s])
        return {"case": c, "sections": s, "q": normal(c["T"], c["Hq"], c["D"]), "k": normal(c["T"], c["Hk"], c["D"]),
                "pos": pos, "freq": freq, "axis": torch.tensor(_axis_of_pair(s), device=DEVICE)}
    n = _lengths(c)
    if c["op"] == "attn":
        cq, ck = _starts([q for q, _ in n]), _starts([k for _, k in n])
        return {"case": c, "q": normal(max(1, cq[-1]), c["Hq"], c["D"])[:cq[-1]], "k": normal(max(1, ck[-1]), c["Hk"], c["D"])[:ck[-1]],
                "v": normal(max(1, ck[-1]), c["Hk"], c["D"])[:ck[-1]], "cu_q": _ints(cq), "cu_k": _ints(ck),
                "max_q": max(q for q, _ in n), "max_k": max(k for _, k in n)}
    if c["op"] == "append":
        kc, vc, scales, table = _cache(c, g, [a + h for a, h in n], 0)
        cu = _starts([a for a, _ in n])
        # what is already there: a last page partly filled, the slots behind it empty
        for b, (a, h) in enumerate(n):
            if h % PAGE:
                at = table[b, h // PAGE].long()
                kc[at, :, h % PAGE:, :] = 0
                vc[at, :, :, h % PAGE:] = 0
        touched = [(b, p) for b, (a, h) in enumerate(n) if a for p in range(h // PAGE, _pages(a + h))]
        return {"case": c, "k": normal(cu[-1], c["Hk"], c["D"]), "v": normal(cu[-1], c["Hk"], c["D"]), "kc": kc, "vc": vc,
                "scales": scales, "table": table, "cu": _ints(cu), "start": _ints([h for _, h in n]),
                "max_new": max(a for a, _ in n), "touched": torch.tensor(touched, device=DEVICE)}
    kc, vc, scales, table = _cache(c, g, n, 0)
    return {"case": c, "q": normal(c["B"], c["Lq"], c["Hq"], c["D"]), "kc": kc, "vc": vc, "scales": scales, "table": table,
            "lens": _ints(n), "max_len": max(n)}


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if own:
        from paper_1606_05688_amd import binding as znni
        if c["op"] == "rope":
            return znni.znni_rope_axes(s["q"], s["k"], s["pos"], s["freq"], s["sections"], pairing=c["pairing"])
        if c["op"] == "attn":
            return znni.znni_attn_window(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["max_q"], s["max_k"],
                                         left=c["left"], right=c["right"], sinks=c["sinks"])
        if c["op"] == "append":
            znni.znni_kv8_append(s["kc"], s["vc"], s["scales"], s["k"], s["v"], s["table"], s["cu"], s["start"], s["max_new"])
            return s["kc"].view(torch.float8_e4m3fn), s["vc"].view(torch.float8_e4m3fn), s["scales"]
        return znni.znni_kv8_attn(s["q"], s["kc"], s["vc"], s["scales"], s["table"], s["lens"], s["max_len"],
                                  left=c["left"], sinks=c["sinks"])
    return {"rope": _plain_rope, "attn": _plain_attn, "append": _plain_append, "kv8": _plain_kv8}[c["op"]](s, c)


def _turn(x, cos, sin, R, pairing):
    x32, cos, sin = x.float(), cos[:, None, :], sin[:, None, :]
    y = x32.clone()
    if pairing == "halves":
        u, v = x32[..., :R], x32[..., R:2 * R]
        y[..., :R] = u * cos - v * sin
        y[..., R:2 * R] = u * sin + v * cos
    else:
        u, v = x32[..., 0:2 * R:2], x32[..., 1:2 * R:2]
        y[..., 0:2 * R:2] = u * cos - v * sin
        y[..., 1:2 * R:2] = u * sin + v * cos
    return y.to(x.dtype)


def _plain_rope(s, c):
    axis = s["axis"]
    angle = s["pos"].float()[:, axis] * s["freq"]
    cos, sin = torch.cos(angle), torch.sin(angle)
    return _turn(s["q"], cos, sin, axis.numel(), c["pairing"]), _turn(s["k"], cos, sin, axis.numel(), c["pairing"])


def _softmax_product(q, k, v, see, scale):
    """q [B][Hk][G*Lq][D], k and v [B][Hk][Lk][D], see [B][1][1][Lq][Lk] -> the rows' weighted sums, zero without weights."""
    B, Hk, rows, D = q.shape
    Lq, Lk = see.shape[-2:]
    w = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(B, Hk, rows // Lq, Lq, Lk)
    w.masked_fill_(~see, -math.inf)
    m = w.amax(-1, keepdim=True)
    w.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = w.sum(-1).view(B, Hk, rows, 1)
    o = torch.matmul(w.view(B, Hk, rows, Lk), v)
    return torch.where(total == 0, torch.zeros_like(o), o / total)


def _plain_attn(s, c):
    Hq, Hk, D, B = c["Hq"], c["Hk"], c["D"], c["B"]
    mq, mk, cq, ck = s["max_q"], s["max_k"], s["cu_q"].long(), s["cu_k"].long()
    nq, nk = cq[1:] - cq[:-1], ck[1:] - ck[:-1]
    i, j = torch.arange(mq, device=DEVICE), torch.arange(mk, device=DEVICE)
    at_q = (cq[:-1, None] + i).clamp(max=max(0, s["q"].shape[0] - 1))
    at_k = (ck[:-1, None] + j).clamp(max=max(0, s["k"].shape[0] - 1))
    p = (nk - nq)[:, None, None] + i[None, :, None]
    key = j[None, None, :]
    see = (key < nk[:, None, None]) & (key <= p + c["right"]) & ((key >= p - c["left"]) | (key < c["sinks"]))
    q = s["q"][at_q].float().view(B, mq, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    k = s["k"][at_k].float().permute(0, 2, 1, 3).contiguous()
    v = s["v"][at_k].float().permute(0, 2, 1, 3).contiguous()
    o = _softmax_product(q, k, v, see[:, None, None], D ** -0.5)
    o = o.view(B, Hq, mq, D)
    token = torch.arange(s["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(cq[1:].contiguous(), token, right=True)
    return o[b, :, token - cq[b]].to(s["q"].dtype)


def _value(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _fill(codes, scales, which, page, x, is_new, is_old, values_first):
    """Pages `page` of a pool with the tokens x [N][PAGE][Hk][D] in the slots is_new [N][PAGE], those of is_old kept."""
    x = x.permute(0, 2, 1, 3).float() if not values_first else x.permute(0, 2, 3, 1).float()
    shape = (-1, 1, PAGE, 1) if not values_first else (-1, 1, 1, PAGE)
    new, old = is_new.view(shape), is_old.view(shape)
    size = torch.where(new & torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax((2, 3))
    m, e = torch.frexp(size)
    e = torch.where(size == 0, torch.full_like(e, -126), e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126)
    before = scales[page][:, :, which]
    held = is_old.any(1, keepdim=True)
    e = torch.where(held, torch.maximum(e, torch.frexp(before)[1] - 1), e)
    scale = torch.ldexp(torch.ones_like(before), e)
    had = codes[page]
    kept = (_value(had) * torch.where(held, before / scale, torch.ones_like(scale))[:, :, None, None])
    y = (x / scale[:, :, None, None])
    y = torch.where(y.abs() > 448, torch.copysign(torch.full_like(y, 448), y), y)
    put = torch.where(new, y, kept).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[page] = torch.where(new | old, put, had)
    scales[page, :, which] = scale


def _plain_append(s, c):
    b, index = s["touched"][:, 0], s["touched"][:, 1]
    page = s["table"][b, index].long()
    cu, start = s["cu"].long(), s["start"].long()
    at = index[:, None] * PAGE + torch.arange(PAGE, device=DEVICE)
    token = at - start[b][:, None]
    is_new, is_old = (token >= 0) & (token < (cu[1:] - cu[:-1])[b][:, None]), token < 0
    token = (token + cu[b][:, None]).clamp(0, s["k"].shape[0] - 1)
    _fill(s["kc"], s["scales"], 0, page, s["k"][token], is_new, is_old, False)
    _fill(s["vc"], s["scales"], 1, page, s["v"][token], is_new, is_old, True)
    return s["kc"].view(torch.float8_e4m3fn), s["vc"].view(torch.float8_e4m3fn), s["scales"]


def _plain_kv8(s, c):
    B, Lq, Hq, D = s["q"].shape
    Hk, table = c["Hk"], s["table"].long()
    n = table.shape[1] * PAGE
    scale = s["scales"][table]
    k = _value(s["kc"][table]).mul_(scale[..., 0, None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hk, n, D)
    v = _value(s["vc"][table]).mul_(scale[..., 1, None, None]).permute(0, 2, 1, 4, 3).reshape(B, Hk, n, D)
    lens = s["lens"].long()[:, None, None]
    key = torch.arange(n, device=DEVICE)[None, None, :]
    p = lens - Lq + torch.arange(Lq, device=DEVICE)[None, :, None]
    see = (key <= p) & ((key >= p - c["left"]) | (key < c["sinks"]))
    q = s["q"].float().view(B, Lq, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    o = _softmax_product(q, k, v, see[:, None, None], D ** -0.5)
    return o.view(B, Hq, Lq, D).transpose(1, 2).to(s["q"].dtype).contiguous()


# ---- 64 bits -------------------------------------------------------------------------------------------------------

def _round_e4m3(y):
    """The nearest value of three mantissa bits, exponents from -6, largest 448; ties to the even one."""
    y = y.clamp(-448.0, 448.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_rows(q, k, v, positions, left, right, sinks):
    """Rows q [n][D] at `positions` against k, v [m][D], one head, in 64 bits."""
    out = torch.zeros_like(q)
    for at in range(0, q.shape[0], 4096):
        p = positions[at:at + 4096, None]
        j = torch.arange(k.shape[0], device=q.device)[None, :]
        see = (j <= p + right) & ((j >= p - left) | (j < sinks))
        score = (q[at:at + 4096] @ k.T) * q.shape[1] ** -0.5
        top = torch.where(see, score, -math.inf).max(1, keepdim=True).values
        weight = torch.where(see, torch.exp(score - torch.where(torch.isinf(top), 0.0, top)), 0.0)
        total = weight.sum(1, keepdim=True)
        out[at:at + 4096] = torch.where(total > 0, (weight @ v) / total, 0.0)
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        R, got = len(s["freq"]), []
        axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEVICE), torch.tensor(s["sections"], device=DEVICE))
        turn = torch.polar(torch.ones((c["T"], R), dtype=torch.float64, device=DEVICE), s["pos"].double()[:, axis] * s["freq"].double())
        for x in (s["q"], s["k"]):
            x = x.double()
            pairs = x[..., :2 * R].unflatten(-1, (2, R)).transpose(-1, -2) if c["pairing"] == "halves" else x[..., :2 * R].unflatten(-1, (R, 2))
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
            z = z.transpose(-1, -2) if c["pairing"] == "halves" else z
            got.append(torch.cat((z.flatten(-2), x[..., 2 * R:]), -1))
        return tuple(got)
    n = _lengths(c)
    if c["op"] == "attn":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        aq = ak = 0
        for lq, lk in n:
            if lq and lk:
                p = torch.arange(lq, device=DEVICE) + (lk - lq)
                for h in range(c["Hq"]):
                    hk = h // (c["Hq"] // c["Hk"])
                    out[aq:aq + lq, h] = _exact_rows(s["q"][aq:aq + lq, h].double(), s["k"][ak:ak + lk, hk].double(),
                                                     s["v"][ak:ak + lk, hk].double(), p, c["left"], c["right"], c["sinks"])
            aq, ak = aq + lq, ak + lk
        return out
    if c["op"] == "append":
        sc = s["scales"].double()
        pools = []
        for which, (pool, x) in enumerate(((s["kc"], s["k"]), (s["vc"], s["v"]))):
            val = pool.view(torch.float8_e4m3fn).double()
            val = val.transpose(2, 3).contiguous() if which else val                 # [page][Hk][PAGE][D]
            at = 0
            for b, (new, have) in enumerate(n):
                done = 0
                while done < new:
                    slot = (have + done) % PAGE
                    page = int(s["table"][b, (have + done) // PAGE])
                    part = x[at + done:at + min(new, done + PAGE - slot)].double().transpose(0, 1)       # [Hk][tokens][D]
                    top = part.abs().amax((1, 2))
                    e = torch.ceil(torch.log2(top / 448)).clamp(min=-126)
                    e = torch.where(448 * torch.exp2(e) < top, e + 1, torch.where(448 * torch.exp2(e - 1) >= top, e - 1, e)).clamp(min=-126)
                    if slot:
                        was = torch.log2(sc[page, :, which])
                        e = torch.maximum(e, was)
                        val[page, :, :slot] = _round_e4m3(val[page, :, :slot] * torch.exp2(was - e)[:, None, None])
                    val[page, :, slot:slot + part.shape[1]] = _round_e4m3(part * torch.exp2(-e)[:, None, None])
                    sc[page, :, which] = torch.exp2(e)
                    done += part.shape[1]
                at += new
            pools.append(val.transpose(2, 3).contiguous() if which else val)
        return pools[0], pools[1], sc
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, l in enumerate(n):
        pages = s["table"][b, :_pages(l)].long()
        for hk in range(c["Hk"] if l else 0):
            k = s["kc"][pages, hk].view(torch.float8_e4m3fn).double() * s["scales"][pages, hk, 0].double()[:, None, None]
            v = s["vc"][pages, hk].view(torch.float8_e4m3fn).double() * s["scales"][pages, hk, 1].double()[:, None, None]
            k, v = k.flatten(0, 1)[:l], v.transpose(1, 2).flatten(0, 1)[:l]
            for h in range(hk * (c["Hq"] // c["Hk"]), (hk + 1) * (c["Hq"] // c["Hk"])):
                p = torch.arange(c["Lq"], device=DEVICE) + (l - c["Lq"])
                out[b, :, h] = _exact_rows(s["q"][b, :, h].double(), k, v, p, c["left"], 0, c["sinks"])
    return out
