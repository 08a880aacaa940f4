"""Timed cases of the operators around the quantized linear layers of a decoder
that keeps its keys and values in MXFP4: block tables and slot maps, rotary
positions with several axes, the cache's write and read-back, and attention
over the cache.

A case is a dict of plain values.  "op" names the operator of one pass:

  assign     rfq_block_assign: blocks, slots and positions of one step's tokens
  release    rfq_block_release: the blocks of requests that ended go back
  rope       rfq_rope, or with "backward" rfq_rope_backward
  append     rfq_kv_append: q rotated, k rotated and quantized, v quantized, both
             into their slots; the written tokens are read back (rfq_kv_gather)
  attention  rfq_kv_attention over block tables

The cache holds, per block of `page` tokens and per key/value head, MXFP4 codes
[page][D / 2] and E8M0 scale bytes [page][D / 32].  The lengths of a case's
requests come from the case alone, the contents from the seed.  Heads of 128
channels times 32 and 40 are the widths 4096 and 5120 of this package's
workloads, 4096, 8192 and 32768 its token counts; the others are generic.

With own false, run computes the plain form: elementary torch operations in 32
bits, rounded once at the end.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # One decode step of 16 requests: every launch's latency counts.
        _blocks("assign_16", "assign", 16, 1, 1, 0, 4096, 16),
        # A batch of 2000 requests that mixes decode and prompts, small pages.
        _blocks("assign_2000_mixed", "assign", 2000, 0, 128, 0, 8000, 16),
        # Requests of every length end together.
        _blocks("release_500", "release", 500, 0, 0, 0, 16000, 32),
        # Queries and keys of a prompt of odd length, positions with three axes.
        _rope("rope_1000", 1000, 40, 128, 128, 3, False, False, "bf16", 4096),
        # A video transformer's whole sequence, the gradient's direction:
        # neighbouring pairs, positions (time, height, width).
        _rope("rope_video_32768_backward", 32768, 40, 128, 128, 3, True, True, "bf16", 1024),
        # Decode of 16 requests: one token each.
        _append("append_16", 16, 32, 8, 128, 128, 1, False, "bf16", 16, 4096),
        # A batch of prompts.
        _append("append_8192", 8192, 32, 8, 128, 128, 3, False, "bf16", 64, 16384),
        # Decode of one request with a short history: the smallest call.
        _attention("decode_1", 1, 1, 1, 700, 700, 32, 8, 128, 16),
        # Decode of a batch whose histories differ widely.
        _attention("decode_64_ragged", 64, 1, 1, 1, 8192, 32, 8, 128, 16),
        # Decode of a few requests over long histories.
        _attention("decode_4_long", 4, 1, 1, 131072, 131072, 40, 8, 128, 64),
        # The last pieces of two long prompts, a window over the past.
        _attention("chunk_2_window", 2, 300, 600, 12000, 16000, 28, 4, 128, 32, window=8192),
        # A whole prompt at once: the largest amount of arithmetic.
        _attention("prefill_8192", 1, 8192, 8192, 8192, 8192, 32, 8, 128, 64),
    ]


def _blocks(name, op, B, new_lo, new_hi, ctx_lo, ctx_hi, page):
    return {"name": name, "op": op, "B": B, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "page": page, "pick": 1}


def _rope(name, T, H, D, rotary, axes, interleaved, backward, x, max_pos):
    return {"name": name, "op": "rope", "T": T, "H": H, "D": D, "rotary": rotary, "axes": axes,
            "interleaved": interleaved, "backward": backward, "x": x, "max_pos": max_pos}


def _append(name, T, Hq, Hkv, D, rotary, axes, interleaved, x, page, max_pos):
    return {"name": name, "op": "append", "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "rotary": rotary,
            "axes": axes, "interleaved": interleaved, "x": x, "page": page, "max_pos": max_pos}


def _attention(name, B, nq_lo, nq_hi, len_lo, len_hi, Hq, Hkv, D, page, causal=True, window=0):
    return {"name": name, "op": "attention", "B": B, "nq_lo": nq_lo, "nq_hi": nq_hi,
            "len_lo": len_lo, "len_hi": len_hi, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "causal": causal, "window": window, "pick": 1}


def draw(rng):
    """One more case: an operator, sizes spread over their logarithms, every
    head width, page, axis count, pairing and type."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["assign", "release", "rope", "rope", "append", "append",
                     "attention", "attention", "attention", "attention"])
    page = rng.choice([16, 32, 64, 128])
    D = rng.choice([64, 128, 128, 256])
    if op in ("assign", "release"):
        case = _blocks("", op, spread(1, 2000), rng.choice([0, 1]), spread(1, 128), 0,
                       spread(16, 16000), page)
        case["pick"] = rng.randrange(1 << 30)
    elif op == "rope":
        H = rng.choice([1, 8, 24, 36, 40])
        T = spread(1, min(32768, 32768 * 40 * 128 // (H * D)))
        case = _rope("", T, H, D, rng.choice([D, D, D // 2]), rng.choice([1, 2, 3]),
                     rng.random() < 0.5, rng.random() < 0.5,
                     "f32" if T * H * D <= 1 << 26 and rng.random() < 0.3 else "bf16",
                     rng.choice([1024, 4096]))
    elif op == "append":
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 4, 5, 7, 8])
        T = spread(1, max(1, min(8192, 8192 * 48 * 128 // ((Hq + 2 * Hkv) * D))))
        case = _append("", T, Hq, Hkv, D, rng.choice([D, D, D // 2]), rng.choice([1, 2, 3]),
                       rng.random() < 0.3, "f32" if T <= 2048 and rng.random() < 0.25 else "bf16",
                       page, 16384)
    else:
        while True:
            Hkv = rng.choice([1, 2, 4, 8])
            G = rng.choice([1, 4, 5, 7, 8, 16])
            nq = 1 if rng.random() < 0.5 else spread(2, 4096)
            B = spread(1, 128) if nq == 1 else spread(1, 8)
            top = spread(max(nq, 16), 100000)
            kv = B * top * Hkv * D
            if kv <= 4 * 131072 * 8 * 128 and B * nq * Hkv * G * top * D <= 32 * 8192 * 8192 * 128:
                break
        even = rng.random() < 0.3
        case = _attention("", B, nq if even else max(1, nq // 2), nq, top if even else nq, top,
                          Hkv * G, Hkv, D, page, causal=nq == 1 or rng.random() < 0.8,
                          window=spread(64, 8192) if rng.random() < 0.25 else 0)
        case["pick"] = rng.randrange(1 << 30)
    del case["name"]
    return case


# ---- the requests of a case (from the case alone)

def _lengths(case):
    """Per request (cached tokens before the step, new tokens): for attention the
    new tokens are among the cached ones.  Lengths are spread over their
    logarithm; a large batch has an idle request."""
    rng = random.Random(case["pick"])

    def spread(lo, hi):
        if lo >= hi:
            return hi
        return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))) - 1)))

    out = []
    for b in range(case["B"]):
        if case["op"] == "attention":
            nq = rng.randint(case["nq_lo"], case["nq_hi"])
            if case["nq_lo"] < case["nq_hi"] and case["B"] > 4 and b == 2:
                nq = 0
            out.append((max(nq, spread(case["len_lo"], case["len_hi"])), nq))
        else:
            out.append((spread(case["ctx_lo"], case["ctx_hi"]),
                        rng.randint(case["new_lo"], case["new_hi"])))
    return out


def _ceil(a, b):
    return -(-a // b)


# ---- inputs

_X = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cos_sin(max_pos, rotary):
    """[max_pos][rotary / 2][2] cosines and sines of p theta_j in float32."""
    theta = 1e6 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    angle = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * theta
    return torch.stack((torch.cos(angle), torch.sin(angle)), -1).float().contiguous()


def _axes(case):
    """The position axis of each rotated pair: contiguous sections for
    neighbouring pairs, alternating for the others."""
    n, half = case["axes"], case["rotary"] // 2
    if case["interleaved"]:
        return bytes(min(n - 1, j * n // half) for j in range(half))
    return bytes(j % n for j in range(half))


def _positions(case, gen):
    """[axes][T] positions: a frame grid where there are three axes (the tokens of
    a video), a running count with a random start for fewer."""
    T, top = case["T"], case["max_pos"]
    i = torch.arange(T, device="cuda")
    first = int(torch.randint(0, max(1, top - T), (1,), generator=gen, device="cuda")) if T < top else 0
    run_ = (first + i) % top
    if case["axes"] < 3:
        return run_.expand(case["axes"], T).int().contiguous()
    side = max(1, min(int(math.sqrt(T)), 40))
    return torch.stack((i // (side * side) % top, i // side % side, i % side)).int().contiguous()


def _prepare_blocks(case, gen):
    lens, page = _lengths(case), case["page"]
    ctx, new = [c for c, _ in lens], [n for _, n in lens]
    held = [_ceil(c, page) for c in ctx]
    extra = sum(_ceil(c + n, page) - _ceil(c, page) for c, n in lens)
    total = sum(held) + extra + 7
    ids = torch.randperm(total, generator=gen, device="cuda").int()
    W = max(_ceil(c + n, page) for c, n in lens) + 1
    tables = torch.full((case["B"], W), -1, dtype=torch.int32, device="cuda")
    h = _ints(held)
    owned = torch.arange(W, device="cuda")[None, :] < h[:, None]
    tables[owned] = ids[:sum(held)]
    state = {"case": case, "ctx": _ints(ctx), "new": _ints(new), "tables": tables}
    free = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    free[:total - sum(held)] = ids[sum(held):]
    state["free"] = free
    state["free_count"] = _ints([total - sum(held)])
    state["tokens"] = sum(new) + 5              # padded as a captured step is
    state["ended"] = (torch.rand(case["B"], generator=gen, device="cuda") < 0.5).to(torch.uint8)
    return state


def _activations(shape, gen):
    """N(0, 1) with two channels of a head ten times larger."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x[..., torch.randperm(shape[-1], generator=gen, device="cuda")[:2]] *= 10.0
    return x


def _cache(blocks, heads, page, D):
    """A cache as it is allocated: codes and scales of unused tokens hold anything,
    here the byte that stands for NaN."""
    def part(width):
        return torch.full((blocks, heads, page, width), 255, dtype=torch.uint8, device="cuda")
    return part(D // 2), part(D // 32), part(D // 2), part(D // 32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    if op in ("assign", "release"):
        return _prepare_blocks(case, gen)
    state = {"case": case, "table": torch.tensor(_E2M1, device="cuda")}
    if op == "attention":
        return _prepare_attention(case, gen, state)
    state["cos_sin"] = _cos_sin(case["max_pos"], case["rotary"])
    state["axes"] = _axes(case)
    state["axis_of"] = torch.tensor(list(state["axes"]), device="cuda")
    state["positions"] = _positions(case, gen)
    T, D = case["T"], case["D"]
    if op == "rope":
        state["x"] = _activations((T, case["H"], D), gen).to(_X[case["x"]])
        return state
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    # One token's q, k and v are one row, as a joint projection writes it.
    qkv = _activations((T, Hq + 2 * Hkv, D), gen).to(_X[case["x"]])
    state["q"], state["k"], state["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    blocks = _ceil(T, page)
    state["cache"] = _cache(blocks, Hkv, page, D)
    order = torch.randperm(blocks, generator=gen, device="cuda")
    i = torch.arange(T, device="cuda")
    state["slots"] = (order[i // page] * page + i % page).int()
    return state


def _prepare_attention(case, gen, state):
    lens, page, Hkv, D = _lengths(case), case["page"], case["Hkv"], case["D"]
    held = [_ceil(n, page) for n, _ in lens]
    blocks = sum(held) + 3
    W = max(1, max(held))
    ids = torch.randperm(blocks, generator=gen, device="cuda").int()
    tables = torch.full((case["B"], W), -1, dtype=torch.int32, device="cuda")
    tables[torch.arange(W, device="cuda")[None, :] < _ints(held)[:, None]] = ids[:sum(held)]
    cache = _cache(blocks, Hkv, page, D)
    # Every slot of the used pages up to the request's length.
    tokens = sum(n for n, _ in lens)
    if tokens:
        n = _ints([n for n, _ in lens])
        b = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), n)
        i = torch.arange(tokens, device="cuda") - (torch.cumsum(n, 0) - n)[b]
        slots = tables[b, i // page].long() * page + i % page
        for at in (0, 2):
            for part in slots.split(1 << 18):
                _store(cache[at], cache[at + 1], part,
                       _activations((part.numel(), Hkv, D), gen) * (0.5 if at else 1.0))
    rows = sum(q for _, q in lens)
    starts = [0]
    for _, q in lens:
        starts.append(starts[-1] + q)
    state.update(cache=cache, tables=tables, seq_lens=_ints([n for n, _ in lens]),
                 starts=_ints(starts), q=torch.randn((rows, case["Hq"], D), device="cuda",
                                                     generator=gen).bfloat16(),
                 max_query=max(1, max(q for _, q in lens)), max_seq=max(1, max(n for n, _ in lens)),
                 scale=D ** -0.5)
    return state


# ---- the plain forms

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _encode(x):
    """MXFP4 codes [.., D / 2] and scale bytes [.., D / 32] of float32 x [.., D]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    e = b.abs().amax(-1).view(torch.int32) >> 23
    byte = (e - 2).clamp(min=0)
    y = b * ((254 - byte) << 23).view(torch.float32)[..., None]     # 2^(127 - byte)
    a = y.abs()
    k = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int()
         + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    c = (k + 8 * torch.signbit(y).int()).reshape(*x.shape[:-1], -1, 2)
    return (c[..., 0] + 16 * c[..., 1]).to(torch.uint8), byte.to(torch.uint8)


def _decode(codes, scales, table):
    """float32 values [.., D] of MXFP4 codes [.., D / 2] and scales [.., D / 32];
    table: the 16 values of a code."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    bits = scales.int() << 23
    factor = torch.where(scales == 0, torch.full_like(bits, 1 << 22), bits).view(torch.float32)
    v = table[c.long()].reshape(*scales.shape, 32) * factor[..., None]
    return torch.where((scales == 255)[..., None], math.nan, v).flatten(-2)


def _store(codes, scales, slots, x):
    """x [n][heads][D] quantized into the slots of a cache."""
    page = codes.shape[2]
    c, s = _encode(x.float())
    at = slots.long()
    codes[at // page, :, at % page] = c
    scales[at // page, :, at % page] = s


def _load(codes, scales, slots, table):
    page = codes.shape[2]
    at = slots.long()
    return _decode(codes[at // page, :, at % page], scales[at // page, :, at % page], table)


def _rotate(x, state, backward=False):
    """float32 x [T][H][D] with its first `rotary` channels rotated, pair j by the
    angle of position axis axes[j]; backward: by the opposite angle."""
    case = state["case"]
    R = case["rotary"]
    pos = state["positions"].long()[state["axis_of"]].T                                # [T][R / 2]
    cs = state["cos_sin"][pos, torch.arange(R // 2, device=x.device)]      # [T][R / 2][2]
    c, s = cs[..., 0][:, None], cs[..., 1][:, None]
    s = -s if backward else s
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((y, x[..., R:]), -1)


def _plain_assign(state):
    case, tables, free = state["case"], state["tables"], state["free"]
    page, T, W = case["page"], state["tokens"], tables.shape[1]
    ctx, new, count = state["ctx"].long(), state["new"].long(), state["free_count"].long()
    held = (ctx + page - 1) // page
    need = (ctx + new + page - 1) // page
    fits = need <= W
    extra = torch.where(fits, need - held, 0)
    incl = torch.cumsum(extra, 0)
    ok = fits & ((extra == 0) | (incl <= count))
    first = incl - extra                              # blocks taken before this request's

    def fresh(n):                                     # the n-th block taken from the list
        return free[(count - 1 - n).clamp(0, free.numel() - 1)].long()

    j = torch.arange(W, device=tables.device)[None, :]
    mine = (j >= held[:, None]) & (j < need[:, None]) & ok[:, None]
    tables.copy_(torch.where(mine, fresh(first[:, None] + j - held[:, None]), tables.long()))
    ends = torch.cumsum(new, 0)
    t = torch.arange(T, device=tables.device)
    b = torch.searchsorted(ends, t, right=True).clamp(max=ctx.numel() - 1)
    inside = t < ends[-1]
    pos = torch.where(inside, ctx[b] + t - (ends - new)[b], 0)
    block = tables[b, (pos // page).clamp(max=W - 1)].long()
    slots = torch.where(inside & ok[b], block * page + pos % page, -1)
    starts = torch.cat((torch.zeros_like(ends[:1]), ends))
    taken = torch.where(ok & (extra > 0), incl, 0).amax()
    counts = torch.stack(((count - taken)[0], ends[-1], (~ok).sum()))
    seq = torch.where(ok, ctx + new, 0)
    return slots.int(), pos.int(), seq.int(), starts.int(), counts.int(), tables


def _plain_release(state):
    tables, free = state["tables"], state["free"]
    page, F = state["case"]["page"], free.numel()
    count = state["free_count"].long()
    n = torch.where(state["ended"] != 0, (state["ctx"].long() + page - 1) // page, 0)
    n = n.clamp(max=tables.shape[1])
    incl = torch.cumsum(n, 0)
    k = torch.arange(F, device=free.device) - count
    b = torch.searchsorted(incl, k, right=True).clamp(max=n.numel() - 1)
    given = tables[b, (k - (incl - n)[b]).clamp(0, tables.shape[1] - 1)]
    free.copy_(torch.where((k >= 0) & (k < incl[-1]), given, free))
    return free, (count + incl[-1]).clamp(max=F).int()


def _visible(case, state, keys):
    """[B][nq][keys] whether query i of request b attends to token j, and the
    queries' rows in q (one past the last where there is no such query)."""
    dev = state["q"].device
    n, starts = state["seq_lens"].long(), state["starts"].long()
    nq = starts[1:] - starts[:-1]
    i = torch.arange(state["max_query"], device=dev)
    j = torch.arange(keys, device=dev)
    pos = (n - nq)[:, None] + i[None, :]
    seen = (j < n[:, None, None]) & (i[None, :, None] < nq[:, None, None])
    if case["causal"]:
        seen = seen & (j <= pos[..., None])
    if case["window"]:
        seen = seen & (j > pos[..., None] - case["window"])
    rows = starts[:-1, None] + i[None, :]
    return seen, torch.where(i[None, :] < nq[:, None], rows, state["q"].shape[0])


def _attend(state):
    """Attention output [rows][Hq][D] and log-sum-exp [rows][Hq] in float32."""
    case, q = state["case"], state["q"]
    B, Hq, Hkv, D, page = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    G, nq, W = Hq // Hkv, state["max_query"], state["tables"].shape[1]
    keys = W * page
    seen, rows = _visible(case, state, keys)
    blocks = state["tables"].long().clamp(min=0)
    kc, ks, vc, vs = state["cache"]

    def whole(codes, scales):                        # [B][Hkv][keys][D]
        x = _decode(codes[blocks], scales[blocks], state["table"])   # [B][W][Hkv][page][D]
        x = x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, keys, D)
        held = torch.arange(keys, device=q.device) < state["seq_lens"][:, None]
        return torch.where(held[:, None, :, None], x, 0.0)

    x = q[rows.clamp(max=q.shape[0] - 1)].float().reshape(B, nq, Hkv, G, D).permute(0, 2, 3, 1, 4)
    s = x.reshape(B, Hkv, G * nq, D) @ whole(kc, ks).transpose(2, 3).contiguous()
    s = s.reshape(B, Hkv, G, nq, keys).mul_(state["scale"])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(B, Hkv, G * nq, keys) @ whole(vc, vs)).reshape(B, Hkv, G, nq, D)
    o = torch.where(total != 0, o / total, 0.0)
    lse = (m + torch.log(total)).squeeze(-1)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, nq, Hq, D)
    lse = lse.permute(0, 3, 1, 2).reshape(B, nq, Hq)
    n = q.shape[0]
    out = o.new_empty(n + 1, Hq, D).index_put_((rows,), o)
    out_lse = lse.new_empty(n + 1, Hq).index_put_((rows,), lse)
    return out[:n], out_lse[:n]


def _plain(state):
    case = state["case"]
    op = case["op"]
    if op == "assign":
        return _plain_assign(state)
    if op == "release":
        return _plain_release(state)
    if op == "rope":
        return _rotate(state["x"].float(), state, case["backward"]).to(state["x"].dtype)
    if op == "append":
        kc, ks, vc, vs = state["cache"]
        _store(kc, ks, state["slots"], _rotate(state["k"].float(), state))
        _store(vc, vs, state["slots"], state["v"].float())
        slots, table = state["slots"], state["table"]
        return (_rotate(state["q"].float(), state).to(state["q"].dtype),
                _load(kc, ks, slots, table).bfloat16(), _load(vc, vs, slots, table).bfloat16())
    out, lse = _attend(state)
    return out.bfloat16(), lse


# ---- one pass

def run(state):
    if not own:
        return _plain(state)
    import paper_2608_26581_amd as rfq
    case = state["case"]
    op = case["op"]
    if op == "assign":
        r = rfq.rfq_block_assign(state["ctx"], state["new"], state["tables"], state["free"],
                                 state["free_count"], case["page"], state["tokens"])
        return (*r, state["tables"])
    if op == "release":
        count = rfq.rfq_block_release(state["ctx"], state["ended"], state["tables"], state["free"],
                                      state["free_count"], case["page"])
        return state["free"], count
    if op == "rope":
        f = rfq.rfq_rope_backward if case["backward"] else rfq.rfq_rope
        return f(state["x"], state["positions"], state["cos_sin"], state["axes"],
                 interleaved=case["interleaved"])
    if op == "append":
        q = rfq.rfq_kv_append(state["k"], state["v"], state["slots"], state["cache"],
                              q=state["q"], positions=state["positions"],
                              cos_sin=state["cos_sin"], axes=state["axes"],
                              interleaved=case["interleaved"])
        return (q, *rfq.rfq_kv_gather(state["cache"], state["slots"]))
    return rfq.rfq_kv_attention(state["q"], state["cache"], state["tables"], state["seq_lens"],
                                state["starts"], state["max_query"], state["max_seq"],
                                scale=state["scale"], causal=case["causal"],
                                window=case["window"], return_lse=True)


# ---- what a pass cannot do without

def work(case):
    op = case["op"]
    mx = 0.5 + 1 / 32
    if op in ("assign", "release"):
        lens, page = _lengths(case), case["page"]
        if op == "release":          # half of the requests end: their blocks are copied
            moved = sum(_ceil(c, page) for c, _ in lens) / 2
            return {"bytes": 5 * case["B"] + 8 * moved, "flops": 0}
        taken = sum(_ceil(c + n, page) - _ceil(c, page) for c, n in lens)
        return {"bytes": 16 * case["B"] + 8 * taken + 8 * sum(n for _, n in lens), "flops": 0}
    if op == "attention":
        lens, D, Hq, Hkv = _lengths(case), case["D"], case["Hq"], case["Hkv"]
        window = case["window"]
        pairs = tokens = rows = 0
        for n, nq in lens:
            if not nq:
                continue
            rows += nq
            first = max(0, n - nq - window + 1) if window else 0
            tokens += n - first
            if not case["causal"]:           # from the window's start to the end
                pairs += nq * n - sum(max(0, n - nq + i - window + 1) for i in range(nq) if window)
            else:
                pairs += sum(min(n - nq + i + 1, window or n) for i in range(nq))
        kv = 2 * tokens * Hkv * D * mx
        return {"bytes": kv + rows * Hq * (2 * 2 * D + 4) + 4 * tokens / case["page"],
                "flops": 4 * pairs * Hq * D}
    T, D = case["T"], case["D"]
    xb = {"bf16": 2, "f32": 4}[case["x"]]
    angles = 4 * case["axes"] * T + min(T, case["max_pos"]) * case["rotary"] * 4
    if op == "rope":
        return {"bytes": 2 * T * case["H"] * D * xb + angles, "flops": 3 * T * case["H"] * case["rotary"]}
    Hq, Hkv = case["Hq"], case["Hkv"]
    return {"bytes": T * D * (2 * Hq * xb + 2 * Hkv * (xb + mx + 2)) + 4 * T + angles,
            "flops": 3 * T * (Hq + Hkv) * case["rotary"]}


# ---- the same values in 64 bits

def _turned(x, case, state, sign):
    """x [T][H][D] in float64, rotated as complex numbers."""
    T, H, R = x.shape[0], x.shape[1], case["rotary"]
    axis = torch.tensor(list(state["axes"]), device=x.device)
    at = torch.gather(state["positions"].long(), 0, axis[:, None].expand(-1, T))    # [R / 2][T]
    cs = state["cos_sin"].double()
    col = torch.arange(R // 2, device=x.device)[:, None].expand(-1, T)
    turn = torch.complex(cs[at, col, 0], sign * cs[at, col, 1]).T[:, None]
    pairs = (x[..., :R].reshape(T, H, R // 2, 2) if case["interleaved"]
             else x[..., :R].reshape(T, H, 2, R // 2).transpose(2, 3))
    z = torch.view_as_real(torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * turn)
    y = z.reshape(T, H, R) if case["interleaved"] else z.transpose(2, 3).reshape(T, H, R)
    return torch.cat((y, x[..., R:]), -1)


def _rounded(x):
    """The values of x's MXFP4 codes in float64."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(-127, 127)
    unit = ((e.long() + 1023) << 52).view(torch.float64)
    a = b.abs() / unit
    step = 0.5 * torch.where(a < 2, 1.0, torch.where(a < 4, 2.0, 4.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.copysign(q * unit, b).reshape(x.shape)


def _values(codes, scales):
    """float64 values of MXFP4 codes, written from the format's bits: sign, two
    bits of exponent (bias 1, zero: subnormal) and one of mantissa."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    exponent, mantissa = (c >> 1) & 3, (c & 1).double()
    v = torch.where(exponent == 0, 0.5 * mantissa,
                    (1 + 0.5 * mantissa) * torch.pow(2.0, (exponent - 1).double()))
    v = torch.where(c >= 8, -v, v)
    unit = ((scales.long() + (1023 - 127)) << 52).view(torch.float64)
    return v * unit.repeat_interleave(32, -1)


def exact(case, seed):
    op = case["op"]
    if op in ("assign", "release"):
        return None                                     # whole numbers
    state = prepare(case, seed)
    if op == "rope":
        return _turned(state["x"].double(), case, state, -1.0 if case["backward"] else 1.0)
    if op == "append":
        return (_turned(state["q"].double(), case, state, 1.0),
                _rounded(_turned(state["k"].double(), case, state, 1.0)),
                _rounded(state["v"].double()))
    # One request, key/value head and piece of its queries at a time.
    lens, page, G = _lengths(case), case["page"], case["Hq"] // case["Hkv"]
    q, tables = state["q"].double(), state["tables"].long()
    out = torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    row = 0
    for b, (n, nq) in enumerate(lens):
        if not nq or not n:
            row += nq
            continue
        pages = tables[b, :_ceil(n, page)]
        for h in range(case["Hkv"]):
            k, v = (_values(c[pages, h].flatten(0, 1)[:n], s[pages, h].flatten(0, 1)[:n])
                    for c, s in (state["cache"][:2], state["cache"][2:]))
            kt = k.T.contiguous()
            for i in range(0, nq, 2048):
                i1 = min(nq, i + 2048)
                pos = torch.arange(n - nq + i, n - nq + i1, device=q.device)[:, None]
                j = torch.arange(n, device=q.device)[None]
                hidden = torch.zeros(i1 - i, n, dtype=torch.bool, device=q.device)
                if case["causal"]:
                    hidden |= j > pos
                if case["window"]:
                    hidden |= j <= pos - case["window"]
                part = q[row + i:row + i1, h * G:(h + 1) * G].transpose(0, 1)
                s = (part.reshape(-1, k.shape[1]) @ kt).reshape(G, i1 - i, n) * state["scale"]
                s.masked_fill_(hidden, -math.inf)
                lse[row + i:row + i1, h * G:(h + 1) * G] = torch.logsumexp(s, -1).T
                o = torch.softmax(s, -1).reshape(-1, n) @ v
                out[row + i:row + i1, h * G:(h + 1) * G] = o.reshape(G, i1 - i, -1).transpose(0, 1)
        row += nq
    return out, lse
