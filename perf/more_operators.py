"""Operators to time around a paged key/value cache that is shared and small: normalising and
rotating queries and keys as they are appended, a cache of 8 bits (written, attended to and read
back), and attention of a batch whose sequences begin with the same tokens.

`run` computes an operator in its plain form from elementary torch operations, or, where `own`
is true, through the package.  `exact` computes the same from the definitions in 64 bits.

The cache's layout (one layer; D = head size, P = tokens per page, U = elements in 16 bytes):
    keys   [page][kv head][P / 16][D / U][16][U]  element d of token t at [t / 16][d / U][t % 16][d % U]
    values [page][kv head][P / 16][2][D][8]       element d of token t at [t / 16][t / 8 % 2][d][t % 8]
    scales [page][kv head][P]                     of keys and of values, where they are held in 8 bits
A cache of 8 bits holds a head's vector x of one token as e4m3 numbers c and a power of two 2^e, with
e = ceil(log2(max |x| / 448)) within the limits of the queries' type, and c = x / 2^e rounded to e4m3,
at most 448.  A sequence's token t lies in page pages[sequence][t / P], at t % P.  The new tokens' rows
of sequence s are starts[s] .. starts[s + 1], its length (the new ones counted) lengths[s].
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LIMITS = {"bf16": (-100, 119), "f16": (-15, 7)}  # of a scale's exponent

BASE = {"dtype": "bf16", "bits": 16, "heads": 32, "kv_heads": 4, "dim": 128, "page": 64, "window": 0, "shared": 0,
        "input": "bf16", "rope_dim": 128, "theta": 1e6, "adjacent": False, "norm": True}


def _case(name, kind, **kw):
    return dict(BASE, name=name, kind=kind, **kw)


def listed():
    return [
        # one decode step of a full batch with norms of queries and keys: latency, 64 scattered tokens
        _case("norm_append_decode64", "append", seqs=64, new_lo=1, new_hi=1, past_lo=100, past_hi=1000),
        # ragged chunks of several prompts; half of each head rotated, adjacent pairs, no shared heads
        _case("norm_append_ragged9", "append", seqs=9, new_lo=1, new_hi=601, past_lo=0, past_hi=1999,
              dtype="f16", input="f16", heads=16, kv_heads=16, dim=64, page=16, rope_dim=32,
              theta=1e4, adjacent=True),
        # the decode step again, held in 8 bits
        _case("append8_decode64", "append", seqs=64, new_lo=1, new_hi=1, past_lo=100, past_hi=1000, bits=8),
        # a long prompt's chunk held in 8 bits, straight from 32-bit projections
        _case("append8_prompt4096", "append", seqs=1, new_lo=4096, new_hi=4096, past_lo=0, past_hi=0,
              input="f32", bits=8),
        # a long context's keys and values, taken out whole
        _case("read8_long1", "read", seqs=1, new_lo=65531, new_hi=65531, past_lo=0, past_hi=0, bits=8),
        # what the last chunks of a ragged batch left, taken out from small pages
        _case("read8_ragged40", "read", seqs=40, new_lo=1, new_hi=900, past_lo=0, past_hi=700, bits=8,
              dtype="f16", heads=16, kv_heads=8, dim=64, page=16),
        # one user, one token, a short context: latency
        _case("attend8_decode1", "attend", seqs=1, new_lo=1, new_hi=1, past_lo=776, past_hi=776, bits=8),
        # a full batch, every context of its own length
        _case("attend8_decode64", "attend", seqs=64, new_lo=1, new_hi=1, past_lo=200, past_hi=16000, bits=8),
        # a chunk of a long prompt behind its earlier chunks: the largest product here
        _case("attend8_chunk4096", "attend", seqs=1, new_lo=4096, new_hi=4096, past_lo=12288, past_hi=12288,
              bits=8),
        # a full batch behind one long system prompt
        _case("shared_decode64", "shared", seqs=64, new_lo=1, new_hi=1, past_lo=50, past_hi=1500, shared=8192),
        # eight answers sampled to one very long document, held in 8 bits
        _case("shared8_decode8", "shared", seqs=8, new_lo=1, new_hi=1, past_lo=10, past_hi=700, shared=65536,
              bits=8),
        # verification windows of five tokens behind a prompt that ends inside a tile
        _case("shared_window24", "shared", seqs=24, new_lo=5, new_hi=5, past_lo=0, past_hi=900, shared=2992,
              dtype="f16", heads=16, kv_heads=2, page=16, rope_dim=64, dim=64),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _fits(case):
    """No more work than the largest listed case of the kind, in a pool and in padded products of
    its order of size (a window leaves most of a pool unread)."""
    last = case["past_hi"] + case["new_hi"]
    rows = case["seqs"] * case["heads"] * case["new_hi"]
    if (case["shared"] + case["seqs"] * last) * case["kv_heads"] * case["dim"] > 1 << 30:
        return False
    if case["kind"] in ("attend", "shared") and rows * (last + case["shared"]) > 1 << 32:
        return False
    w = work(case)
    most = [work(c) for c in listed() if c["kind"] == case["kind"]]
    return all(w[k] <= max(m[k] for m in most) for k in w)


def draw(rng):
    while True:
        kind = rng.choice(["append", "read", "attend", "shared"])
        dtype, dim = rng.choice(["bf16", "f16"]), rng.choice([64, 128, 128, 256])
        kv, page = rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 128])
        form = rng.choice(["token", "window", "chunks"])
        seqs = _log_uniform(rng, 1 if kind != "shared" else 2, 64 if form != "chunks" else 12)
        new = {"token": 1, "window": rng.randint(2, 8)}.get(form)
        new = new or _log_uniform(rng, 9, 256 if kind == "shared" else 2048)
        past = _log_uniform(rng, 1, {"append": 8192, "read": 8192, "attend": 131072, "shared": 2048}[kind])
        bits = rng.choice([8, 16]) if kind in ("read", "shared") else 8
        case = {"kind": kind, "dtype": dtype, "dim": dim, "kv_heads": kv,
                "heads": kv * rng.choice([1, 2, 4, 5, 8]), "page": page,
                "bits": rng.choice([8, 8, 16]) if kind == "append" else bits,
                "window": rng.choice([0, 0, _log_uniform(rng, 100, 4096)]) if kind == "attend" else 0,
                "shared": page * _log_uniform(rng, 1, 65536 // page) if kind == "shared" else 0,
                "input": rng.choice([dtype, "f32"]) if kind == "append" else dtype,
                "rope_dim": rng.choice([dim, dim // 2]), "theta": rng.choice([1e4, 1e6]),
                "adjacent": rng.random() < 0.5, "seqs": seqs,
                "new_lo": new if form != "chunks" else rng.randint(1, new), "new_hi": new,
                "past_lo": rng.randint(0, past), "past_hi": past}
        case["norm"] = kind == "append" and (case["bits"] == 16 or rng.random() < 0.5)
        if _fits(case):
            return case


def _lengths(case):
    """(new tokens, own tokens before them) of every sequence, from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    return [(rng.randint(case["new_lo"], case["new_hi"]), rng.randint(case["past_lo"], case["past_hi"]))
            for _ in range(case["seqs"])]


def _visible(first, last, window):
    """Sum over positions first .. last - 1 of the keys that a token there sees."""
    total = lambda n: n * (n + 1) // 2  # noqa: E731
    pairs = total(last) - total(first)
    if window:
        over = lambda n: total(max(0, n - window))  # noqa: E731
        pairs -= over(last) - over(first)
    return pairs


def work(case):
    hq, hk, d, s, w = (case[k] for k in ("heads", "kv_heads", "dim", "shared", "window"))
    lengths = _lengths(case)
    new = sum(n for n, _ in lengths)
    held = 2 * hk * (d + 1 if case["bits"] == 8 else 2 * d)  # bytes of a token in the cache
    if case["kind"] == "append":
        size = 4 if case["input"] == "f32" else 2
        return {"bytes": new * ((hq + 2 * hk) * d * size + hq * d * 2 + held),
                "flops": new * (hq + hk) * (case["rope_dim"] * 3 + case["norm"] * d * 4)}
    if case["kind"] == "read":
        return {"bytes": new * (held + 4 * hk * d), "flops": new * 2 * hk * d}
    keys = s + sum(min(n + p, n + w - 1) if w else n + p for n, p in lengths)
    pairs = s * new + sum(_visible(p, n + p, w) for n, p in lengths)
    return {"bytes": 4 * new * hq * d + keys * held, "flops": 4 * d * hq * pairs}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s, t=torch.float32: torch.randn(*s, generator=g, device="cuda", dtype=t)  # noqa: E731
    t, hq, hk, d, page = TYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"], case["page"]
    lengths, shared, held = _lengths(case), case["shared"], case["bits"] == 8
    new, total = [n for n, _ in lengths], [shared + n + p for n, p in lengths]
    front = shared // page  # pages of the tokens that all sequences begin with
    counts = [-(-x // page) - front for x in total]
    n_pages, width = front + sum(counts) + 3, front + max(counts)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    pages = torch.zeros(len(total), width, dtype=torch.int32)
    pages[:, :front] = order[:front]
    at = front
    for s, c in enumerate(counts):  # every sequence's pages lie anywhere in the pool
        pages[s, front:front + c] = order[at:at + c]
        at += c
    state = {"case": case, "pages": pages.cuda(), "most_new": max(new), "tokens": sum(new)}
    if front:
        state["prefix"] = order[:front].cuda()
        state["shared"] = torch.tensor([shared], dtype=torch.int32, device="cuda")
    state["starts"] = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    state["lengths"] = torch.tensor(total, dtype=torch.int32, device="cuda")
    if held:
        code = lambda *s: (128.0 * randn(*s, t=t)).clamp_(-448, 448).to(torch.float8_e4m3fn)  # noqa: E731
        scale = lambda: torch.randint(119, 122, (n_pages, hk, page), generator=g, device="cuda",  # noqa: E731
                                      dtype=torch.uint8).view(torch.float8_e8m0fnu)
        state["keys"], state["values"] = code(n_pages, hk, page // 16, d // 16, 16, 16), code(n_pages, hk, page // 16, 2, d, 8)
        state["key_scales"], state["value_scales"] = scale(), scale()
    else:
        state["keys"] = randn(n_pages, hk, page // 16, d // 8, 16, 8, t=t)
        state["values"] = randn(n_pages, hk, page // 16, 2, d, 8, t=t)
    half = case["rope_dim"] // 2
    state["freqs"] = torch.tensor([case["theta"] ** (-i / half) for i in range(half)], dtype=torch.float64,
                                  device="cuda")
    kind, tokens = TYPES[case["input"]], sum(new)
    if case["kind"] != "read":
        state["q"] = (2.0 * randn(tokens, hq, d)).to(kind)
    if case["kind"] == "append":
        state["k"], state["v"] = randn(tokens, hk, d, t=kind), randn(tokens, hk, d, t=kind)
        state["q_norm"] = state["k_norm"] = None
        if case["norm"]:
            state["q_norm"], state["k_norm"] = (1.0 + 0.2 * randn(d)).to(t), (1.0 + 0.2 * randn(d)).to(t)
    if own:
        from paper_2607_09686_amd import KvCache
        scales = {k: state[k][None] for k in ("key_scales", "value_scales")} if held else {}
        state["cache"] = KvCache(n_layers=1, n_heads=hq, n_kv_heads=hk, head_dim=d, page_tokens=page,
                                 n_pages=n_pages, dtype=t, rope_theta=case["theta"],
                                 rope_dim=min(case["rope_dim"], d), rope_adjacent=case["adjacent"],
                                 window=case["window"], keys=state["keys"][None], values=state["values"][None],
                                 storage=torch.float8_e4m3fn if held else None, **scales)
    return state


def run(state):
    return {"append": _append, "read": _read, "attend": _attend, "shared": _shared}[state["case"]["kind"]](state)


EPS = 1e-6


def _place(state):
    """(page, place in it) of every new token, and its position."""
    page = state["case"]["page"]
    rows = torch.arange(state["tokens"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(state["starts"], rows, right=True) - 1
    position = state["lengths"][seq] - state["starts"][seq + 1] + rows
    return state["pages"][seq, (position // page).long()].long(), (position % page).long(), position


def _pools(state):
    names = ("keys", "values", "key_scales", "value_scales") if state["case"]["bits"] == 8 else ("keys", "values")
    return {k: state[k] for k in names}


def _hold(x, dtype):
    """(codes, exponents + 127) of vectors along the last dimension."""
    f, e = torch.frexp(x.abs().amax(-1))
    lo, hi = LIMITS[dtype]
    e = (e - 9 + (f > 0.875)).clamp(lo, hi)
    return torch.ldexp(x, -e[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _append(state):
    case = state["case"]
    if own:
        q = state["cache"].append(state["k"], state["v"], state["pages"], state["starts"], state["lengths"],
                                  q=state["q"], q_norm=state["q_norm"], k_norm=state["k_norm"], norm_eps=EPS)
        return dict(_pools(state), q=q)
    t, r = TYPES[case["dtype"]], case["rope_dim"]
    where, at, position = _place(state)
    angle = position.double()[:, None] * state["freqs"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        y = x.clone()
        a, b = (slice(0, r, 2), slice(1, r, 2)) if case["adjacent"] else (slice(0, r // 2), slice(r // 2, r))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y

    q, k, v = turned(state["q"], state["q_norm"]).to(t), turned(state["k"], state["k_norm"]), state["v"].float()
    tokens, hk, d = k.shape
    if case["bits"] == 8:
        (k, ke), (v, ve) = _hold(k, case["dtype"]), _hold(v, case["dtype"])
        state["key_scales"].view(torch.uint8)[where, :, at] = ke
        state["value_scales"].view(torch.uint8)[where, :, at] = ve
        keys, values, k, v = (x.view(torch.uint8) for x in (state["keys"], state["values"], k, v))
    else:
        keys, values, k, v = state["keys"], state["values"], k.to(t), v.to(t)
    unit = keys.shape[-1]
    keys[where, :, at // 16, :, at % 16] = k.view(tokens, hk, d // unit, unit)
    values[where, :, at // 16, at // 8 % 2, :, at % 8] = v
    return dict(_pools(state), q=q)


def _read(state):
    case = state["case"]
    if own:
        k, v = state["cache"].read(state["tokens"], state["pages"], state["starts"], state["lengths"])
        return {"k": k, "v": v}
    t = TYPES[case["dtype"]]
    where, at, _ = _place(state)
    if case["bits"] == 16:
        k = state["keys"][where, :, at // 16, :, at % 16].flatten(2)
        return {"k": k, "v": state["values"][where, :, at // 16, at // 8 % 2, :, at % 8]}
    keys, values = state["keys"].view(torch.uint8), state["values"].view(torch.uint8)
    k = keys[where, :, at // 16, :, at % 16].flatten(2).view(torch.float8_e4m3fn).float()
    v = values[where, :, at // 16, at // 8 % 2, :, at % 8].view(torch.float8_e4m3fn).float()
    ke, ve = (state[n].view(torch.uint8)[where, :, at].int()[..., None] - 127 for n in ("key_scales", "value_scales"))
    return {"k": torch.ldexp(k, ke).to(t), "v": torch.ldexp(v, ve).to(t)}


def _gathered(state, pages):
    """Keys and values of pages [..., n] as fp32 [..., kv heads, n * page, dim]."""
    case = state["case"]
    span, f = pages.shape[-1] * case["page"], pages.dim() - 1
    front = list(range(f))
    pages = pages.long()
    if case["bits"] == 8:
        k, v = (state[n].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float() for n in ("keys", "values"))
        ke, ve = (torch.ldexp(torch.ones((), device="cuda"), state[n].view(torch.uint8)[pages].int() - 127)
                  for n in ("key_scales", "value_scales"))
        ke, ve = (x.permute(front + [f + 1, f, f + 2]).flatten(-2)[..., None] for x in (ke, ve))
    else:
        k, v = state["keys"][pages].float(), state["values"][pages].float()
    hk, d = k.shape[f + 1], case["dim"]
    k = k.permute(front + [f + 1, f, f + 2, f + 4, f + 3, f + 5])
    v = v.permute(front + [f + 1, f, f + 2, f + 3, f + 5, f + 4])
    shape = tuple(pages.shape[:-1]) + (hk, span, d)
    k, v = k.reshape(shape), v.reshape(shape)
    return (k.mul_(ke), v.mul_(ve)) if case["bits"] == 8 else (k, v)


def _rows(state):
    """The new tokens' rows, padded: their numbers [seqs, most], whether they are there, positions."""
    count = state["starts"][1:] - state["starts"][:-1]
    j = torch.arange(state["most_new"], device="cuda")
    real = j < count[:, None]
    row = (state["starts"][:-1, None] + j).clamp_max(state["tokens"] - 1)
    return row, real, (state["lengths"] - count)[:, None] + j


def _attend(state):
    case = state["case"]
    if own:
        return state["cache"].attend(state["q"], state["pages"], state["starts"], state["lengths"])
    hq, hk, d, most, seqs = case["heads"], case["kv_heads"], case["dim"], state["most_new"], case["seqs"]
    group = hq // hk
    k, v = _gathered(state, state["pages"])
    span = k.shape[2]
    at = torch.arange(span, device="cuda")
    row, real, position = _rows(state)
    q = state["q"][row].view(seqs, most, hk, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hk, group * most, d)
    s = torch.matmul(q.float(), k.transpose(2, 3).contiguous()).mul_(d ** -0.5)
    seen = (at <= position[..., None]) & real[..., None]
    if case["window"]:
        seen &= at > position[..., None] - case["window"]
    s = s.view(seqs, hk, group, most, span).masked_fill_(~seen[:, None, None], float("-inf"))
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(seqs, hk, group * most, span), v).view(seqs, hk, group, most, d) / total
    return o.permute(0, 3, 1, 2, 4).reshape(seqs, most, hq, d)[real].to(TYPES[case["dtype"]])


def _shared(state):
    case = state["case"]
    if own:
        q = state["q"].to(TYPES[case["dtype"]])  # a case's projections may come in another type
        return state["cache"].attend(q, state["pages"], state["starts"], state["lengths"],
                                     prefix=state["prefix"], shared=state["shared"])
    hq, hk, d, most, seqs = case["heads"], case["kv_heads"], case["dim"], state["most_new"], case["seqs"]
    group, tokens = hq // hk, state["tokens"]
    # what all rows see, once for all
    k, v = _gathered(state, state["prefix"])
    q = state["q"].view(tokens, hk, group, d).permute(1, 0, 2, 3).reshape(hk, tokens * group, d)
    p = torch.matmul(q.float(), k.transpose(1, 2).contiguous()).mul_(d ** -0.5)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    first = [x.view(hk, tokens, group, -1).permute(1, 0, 2, 3) for x in (top, p.sum(-1, keepdim=True), torch.matmul(p, v))]
    # what follows it, by sequence
    k, v = _gathered(state, state["pages"][:, case["shared"] // case["page"]:])
    span = k.shape[2]
    at = case["shared"] + torch.arange(span, device="cuda")
    row, real, position = _rows(state)
    q = state["q"][row].view(seqs, most, hk, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hk, group * most, d)
    s = torch.matmul(q.float(), k.transpose(2, 3).contiguous()).mul_(d ** -0.5)
    seen = (at <= position[..., None]) & real[..., None]
    s = s.view(seqs, hk, group, most, span).masked_fill_(~seen[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    o = torch.matmul(p.view(seqs, hk, group * most, span), v).view(seqs, hk, group, most, d)
    after = [x.permute(0, 3, 1, 2, 4)[real] for x in (top, p.sum(-1, keepdim=True), o)]
    top = torch.maximum(first[0], after[0])
    a, b = (first[0] - top).exp(), (after[0] - top).exp()
    o = (a * first[2] + b * after[2]) / (a * first[1] + b * after[1])
    return o.reshape(tokens, hq, d).to(TYPES[case["dtype"]])


def exact(case, seed):
    state = prepare(case, seed)
    return {"append": _exact_append, "read": _exact_read}.get(case["kind"], _exact_attend)(state)


def _exact_scales(scales):
    return torch.exp2(scales.view(torch.uint8).double() - 127)


def _exact_append(state):
    case = state["case"]
    page, r, half, held = case["page"], case["rope_dim"], case["rope_dim"] // 2, case["bits"] == 8
    starts, lengths, pages = (state[k].tolist() for k in ("starts", "lengths", "pages"))
    keys, values = state["keys"].double(), state["values"].double()
    out = {"keys": keys, "values": values}
    if held:
        out["key_scales"], out["value_scales"] = (_exact_scales(state[n]) for n in ("key_scales", "value_scales"))
    q, k, v = state["q"].double(), state["k"].double(), state["v"].double()
    out["q"] = q
    for x, weight in ((q, state["q_norm"]), (k, state["k_norm"])):
        if weight is not None:
            x /= torch.sqrt((x * x).sum(2, keepdim=True) / case["dim"] + EPS)
            x *= weight.double()
    freq = torch.tensor([case["theta"] ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
    lo_e, hi_e = LIMITS[case["dtype"]]
    for s, length in enumerate(lengths):
        lo, hi = starts[s], starts[s + 1]
        position = torch.arange(length - (hi - lo), length, device="cuda")
        turn = torch.exp(1j * position.double()[:, None] * freq)
        for x in (q, k):
            part = x[lo:hi, :, :r]
            pair = part.unflatten(2, (half, 2)) if case["adjacent"] else part.unflatten(2, (2, half)).transpose(2, 3)
            z = torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * turn[:, None]
            pair = torch.view_as_real(z)
            x[lo:hi, :, :r] = (pair if case["adjacent"] else pair.transpose(2, 3)).flatten(2)
        table = torch.tensor(pages[s], device="cuda")[position // page]
        at = position % page
        for x, pool, name in ((k, keys, "key_scales"), (v, values, "value_scales")):
            x = x[lo:hi]
            if held:  # unrounded numbers behind a rounded scale
                scale = torch.exp2(torch.ceil(torch.log2(x.abs().amax(2) / 448)).clamp(lo_e, hi_e))
                out[name][table, :, at] = scale
                x = x / scale[..., None]
            if pool is keys:
                keys[table, :, at // 16, :, at % 16] = x.unflatten(2, (-1, keys.shape[-1]))
            else:
                values[table, :, at // 16, at // 8 % 2, :, at % 8] = x
    return out


def _exact_sequence(state, s, h, length):
    """Keys and values [length, dim] of one sequence and KV head, in 64 bits."""
    d, table = state["case"]["dim"], state["pages"][s, :-(-length // state["case"]["page"])].long()
    held = state["case"]["bits"] == 8
    raw = lambda n: state[n].view(torch.uint8)[table, h] if held else state[n][table, h]  # noqa: E731
    k, v = raw("keys"), raw("values")
    if held:
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    k, v = k.transpose(2, 3).reshape(-1, d).double(), v.transpose(3, 4).reshape(-1, d).double()
    if held:
        k *= _exact_scales(raw("key_scales")).reshape(-1, 1)
        v *= _exact_scales(raw("value_scales")).reshape(-1, 1)
    return k[:length], v[:length]


def _exact_read(state):
    case = state["case"]
    starts, lengths = state["starts"].tolist(), state["lengths"].tolist()
    k = torch.empty(state["tokens"], case["kv_heads"], case["dim"], dtype=torch.float64, device="cuda")
    v = torch.empty_like(k)
    for s, length in enumerate(lengths):
        lo, hi = starts[s], starts[s + 1]
        for h in range(case["kv_heads"]):
            whole = _exact_sequence(state, s, h, length)
            k[lo:hi, h], v[lo:hi, h] = (x[length - (hi - lo):] for x in whole)
    return {"k": k, "v": v}


def _exact_attend(state):
    case = state["case"]
    group = case["heads"] // case["kv_heads"]
    starts, lengths = state["starts"].tolist(), state["lengths"].tolist()
    out = torch.empty(state["q"].shape, dtype=torch.float64, device="cuda")
    for s, length in enumerate(lengths):
        lo, hi = starts[s], starts[s + 1]
        position = torch.arange(length - (hi - lo), length, device="cuda")
        at = torch.arange(length, device="cuda")
        hidden = at > position[:, None]
        if case["window"]:
            hidden |= at <= position[:, None] - case["window"]
        for h in range(case["kv_heads"]):
            k, v = _exact_sequence(state, s, h, length)
            kt = k.t().contiguous()
            for i in range(h * group, (h + 1) * group):
                x = state["q"][lo:hi, i].double().contiguous() @ kt / math.sqrt(case["dim"])
                out[lo:hi, i] = torch.softmax(x.masked_fill_(hidden, -math.inf), 1) @ v
    return out
