"""Timed cases of a layer whose MLP is a set of experts, on RFQ products: the
choice of each token's experts with its weights and gradient, the tokens sorted
by expert, the product with a weight matrix per expert, and the way to the sorted
rows and back with its gradients.

A case is a dict of plain values.  "op" names the operator of one pass:

  route     rfq_route, or with "backward" rfq_route_backward
  sort      rfq_expert_sort: offsets, rows and slots of all (token, choice) pairs
  product   rfq_gemm_experts on MXFP4 codes (primary, or primary and residual)
  gather    rfq_expert_gather: the sorted rows
  combine   rfq_expert_combine, or with "backward" rfq_expert_combine_backward

T tokens choose k of "all" experts; a device holds the E of them from "first" on
(all of them, or its share of a layer split over devices, where the other pairs
are dropped).  Some experts are chosen more often than others.  4096, 12288 and
8192 are sizes of this package's workloads, the others generic.

With own false, run computes the plain form: elementary torch operations in 32
bits, rounded once at the end.
"""
import math

import torch

own = False


def listed():
    return [
        # One decode step of 16 requests: every launch's latency counts.
        _route("route_16", 16, 128, 8, True, "bf16"),
        # A batch of prompts: masked experts and padded tokens, softmax over all.
        _route("route_32768_masked", 32768, 160, 6, False, "f32", masked=True),
        # The gradient of a training batch; a number of experts that is no power of two.
        _route("route_backward_8192", 8192, 60, 4, False, "bf16", backward=True),
        # Decode: two hundred pairs.
        _sort("sort_25", 25, 128, 8),
        # A batch of prompts over many experts.
        _sort("sort_32768", 32768, 256, 8),
        # Decode of 16 requests: bound by the weights of the experts that were chosen.
        _product("product_decode_16", 16, 128, 8, 2048, 1536, True, "bf16"),
        # A short prompt's second product, from sorted rows: odd lengths, plain MXFP4.
        _product("product_down_701", 701, 60, 4, 1408, 2048, False, "f32", mapped=False),
        # A device's half of the experts in a batch of prompts.
        _product("product_half_8192", 8192, 128, 8, 2048, 1536, True, "bf16", E=64, first=64),
        # Few large experts: the largest amount of arithmetic.
        _product("product_8_4096", 4096, 8, 2, 4096, 12288, True, "bf16"),
        # The sorted rows of a batch as a training step makes them.
        _exchange("gather_4096", "gather", 4096, 64, 6, 2048, "bf16"),
        # Decode: the experts' results of 64 requests summed.
        _exchange("combine_64", "combine", 64, 128, 8, 2048, "bf16"),
        # A training step's gradients of the experts' results and of the weights.
        _exchange("combine_backward_8192", "combine", 8192, 128, 8, 2048, "bf16", backward=True),
    ]


def _route(name, T, E, k, renormalize, x, masked=False, backward=False):
    return {"name": name, "op": "route", "T": T, "all": E, "k": k, "renormalize": renormalize,
            "x": x, "masked": masked, "backward": backward}


def _sort(name, T, all_, k, E=None, first=0):
    return {"name": name, "op": "sort", "T": T, "all": all_, "k": k, "E": E or all_, "first": first}


def _product(name, T, all_, k, K, N, residual, z, E=None, first=0, mapped=True):
    return {"name": name, "op": "product", "T": T, "all": all_, "k": k, "E": E or all_,
            "first": first, "K": K, "N": N, "residual": residual, "z": z, "mapped": mapped}


def _exchange(name, op, T, all_, k, N, x, E=None, first=0, backward=False):
    return {"name": name, "op": op, "T": T, "all": all_, "k": k, "E": E or all_, "first": first,
            "N": N, "x": x, "backward": backward}


def draw(rng):
    """One more case: an operator, sizes spread over their logarithms, every type,
    whole layers and shares of layers."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["route", "route", "sort", "product", "product", "product", "product",
                     "gather", "combine", "combine"])
    all_ = rng.choice([8, 16, 60, 64, 128, 160, 256])
    k = rng.choice([1, 2, 4, 6, 8])
    x = rng.choice(["bf16", "bf16", "f32"])
    E, first = all_, 0
    if rng.random() < 0.3:
        E = max(1, all_ // rng.choice([2, 4, 8]))
        first = E * rng.randrange(all_ // E)
    if op == "route":
        case = _route("", spread(1, 32768), all_, k, rng.random() < 0.5, x,
                      masked=rng.random() < 0.3, backward=rng.random() < 0.4)
    elif op == "sort":
        case = _sort("", spread(1, 32768), all_, k, E, first)
    elif op == "product":
        while True:
            T, K, N = spread(1, 16384), 32 * spread(8, 200), spread(64, 8192)
            if T * k * N * K <= 8192 * 12288 * 4096 and E * N * K <= 8 * 12288 * 4096:
                break
        if rng.random() < 0.7:
            N = max(64, N // 64 * 64)
        case = _product("", T, all_, k, K, N, rng.random() < 0.7, rng.choice(["bf16", "bf16", "f32"]),
                        E, first, mapped=rng.random() < 0.6)
    else:
        N = spread(64, 8192)
        if rng.random() < 0.8:
            N = max(64, N // 64 * 64)
        T = spread(1, max(1, min(16384, 8192 * 8 * 2048 // (N * k) // (2 if x == "f32" else 1))))
        case = _exchange("", op, T, all_, k, N, x, E, first,
                         backward=op == "combine" and rng.random() < 0.5)
    del case["name"]
    return case


# ---- inputs

_X = {"bf16": torch.bfloat16, "f32": torch.float32}


def _logits(case, gen):
    """Router logits [T][all]: some experts are liked more than others."""
    T, E = case["T"], case["all"]
    l = torch.randn((T, E), generator=gen, device="cuda")
    l += 0.5 * torch.randn((E,), generator=gen, device="cuda")
    if case.get("masked"):
        # Experts that are out of service, and tokens that are padding.
        l[:, torch.rand((E,), generator=gen, device="cuda") < 0.2] = -math.inf
        l[torch.rand((T,), generator=gen, device="cuda") < 0.05] = -math.inf
    return l


def _choices(case, gen):
    """int32 [T][k] experts."""
    return torch.topk(_logits(case, gen), case["k"], dim=1).indices.int()


def _activations(shape, gen):
    """N(0, 1) with one channel in 200 fifty times larger."""
    x = torch.randn(shape, device="cuda", generator=gen)
    n = max(1, shape[-1] // 200)
    x[..., torch.randperm(shape[-1], generator=gen, device="cuda")[:n]] *= 50.0
    return x


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = {"case": case}
    op, T, k = case["op"], case["T"], case["k"]
    if op == "route":
        state["logits"] = _logits(case, gen).to(_X[case["x"]])
        if case["backward"]:
            state["weights"], state["experts"] = _plain_route(state)
            state["dweights"] = torch.randn((T, k), generator=gen, device="cuda")
        return state
    experts = _choices(case, gen)
    if op == "sort":
        state["experts"] = experts
        return state
    offsets, rows, slots = _sorted(experts, case["E"], case["first"])
    P = T * k
    state.update(offsets=offsets, rows=rows, slots=slots)
    if op == "product":
        K, N, E = case["K"], case["N"], case["E"]
        M = T if case["mapped"] else P
        state["table"] = torch.tensor(_E2M1, device="cuda")
        x = _activations((M, K), gen)
        q = _encode(x)
        state["a"] = (*q, *((_encode(x - _decode(*q, state["table"])) if case["residual"]
                             else (None, None))))
        del x
        w = [_encode(0.02 * torch.randn((N, K), generator=gen, device="cuda")) for _ in range(E)]
        state["w"] = tuple(torch.stack(p) for p in zip(*w))
        # The layer's buffer: rows past the last pair keep what they hold.
        state["z"] = torch.zeros((P, N), dtype=_X[case["z"]], device="cuda")
        return state
    dtype = _X[case["x"]]
    if op == "gather":
        state["x"] = _activations((T, case["N"]), gen).to(dtype)
        return state
    state["z"] = torch.randn((P, case["N"]), generator=gen, device="cuda").to(dtype)
    state["weights"] = torch.softmax(torch.randn((T, k), generator=gen, device="cuda"), -1)
    if case["backward"]:
        state["dout"] = torch.randn((T, case["N"]), generator=gen, device="cuda").to(dtype)
    return state


# ---- the plain forms

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _encode(x):
    """MXFP4 codes [.., K / 2] and scale bytes [.., K / 32] of float32 x [.., K]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    e = b.abs().amax(-1).view(torch.int32) >> 23
    byte = (e - 2).clamp(min=0)
    y = b * ((254 - byte) << 23).view(torch.float32)[..., None]     # 2^(127 - byte)
    a = y.abs()
    c = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int()
         + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    c = (c + 8 * torch.signbit(y).int()).reshape(*x.shape[:-1], -1, 2)
    return (c[..., 0] + 16 * c[..., 1]).to(torch.uint8), byte.to(torch.uint8)


def _decode(codes, scales, table):
    """float32 values [.., K] of codes [.., K / 2] and scales [.., K / 32]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    bits = scales.int() << 23
    factor = torch.where(scales == 0, torch.full_like(bits, 1 << 22), bits).view(torch.float32)
    return (table[c.long()].reshape(*scales.shape, 32) * factor[..., None]).flatten(-2)


def _sorted(experts, E, first):
    """offsets [E + 1], rows [T k] (-1 past the last) and slots [T][k] (-1: dropped)."""
    T, k = experts.shape
    e = experts.flatten().long() - first
    e = torch.where((e >= 0) & (e < E), e, E)
    order = torch.sort(e, stable=True).indices
    key = e[order]
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=e.device))
    held = key < E
    rows = torch.where(held, order // k, -1)
    slots = torch.empty_like(order)
    slots[order] = torch.where(held, torch.arange(T * k, device=e.device), -1)
    return offsets.int(), rows.int(), slots.reshape(T, k).int()


def _plain_route(state):
    case = state["case"]
    l = state["logits"].float()
    v, i = torch.sort(l, dim=1, descending=True, stable=True)
    v, i = v[:, :case["k"]], i[:, :case["k"]]
    hidden = v == -math.inf
    m = torch.where(hidden[:, :1], 0.0, v[:, :1])
    p = torch.exp(v - m)
    total = (p if case["renormalize"] else torch.exp(l - m)).sum(1, keepdim=True)
    return torch.where(hidden, 0.0, p / total), torch.where(hidden, -1, i).int()


def _plain_route_backward(state):
    case, l = state["case"], state["logits"].float()
    w, d, i = state["weights"], state["dweights"], state["experts"].long()
    g = w * d
    s = g.sum(1, keepdim=True)
    if case["renormalize"]:
        out = torch.zeros_like(l)
        g = g - w * s
    else:
        m = l.amax(1, keepdim=True)
        p = torch.exp(l - torch.where(m == -math.inf, 0.0, m))
        total = p.sum(1, keepdim=True)
        out = -torch.where(total != 0, p / total, 0.0) * s
    return out.scatter_add(1, i.clamp(min=0), torch.where(i >= 0, g, 0.0)).to(state["logits"].dtype)


def _plain_product(state):
    a, (wc, ws), table, z = state["a"], state["w"], state["table"], state["z"]
    ends = state["offsets"].tolist()
    parts = [_decode(*a[i:i + 2], table) for i in (0, 2) if a[i] is not None]
    if state["case"]["mapped"]:
        rows = state["rows"][:ends[-1]].long()
        parts = [x[rows] for x in parts]
    for e in range(len(ends) - 1):
        i, j = ends[e], ends[e + 1]
        if i < j:
            w = _decode(wc[e], ws[e], table).T
            s = parts[0][i:j] @ w
            if len(parts) > 1:
                s += parts[1][i:j] @ w
            z[i:j] = s
    return z


def _taken(state):
    """float32 [T][k][N] rows of z, zeros for dropped pairs."""
    s = state["slots"].long()
    return torch.where((s >= 0)[..., None], state["z"][s.clamp(min=0)].float(), 0.0)


def _plain(state):
    case = state["case"]
    op = case["op"]
    if op == "route":
        return _plain_route_backward(state) if case["backward"] else _plain_route(state)
    if op == "sort":
        return _sorted(state["experts"], case["E"], case["first"])
    if op == "product":
        return _plain_product(state)
    if op == "gather":
        r = state["rows"].long()
        return torch.where((r >= 0)[:, None], state["x"][r.clamp(min=0)], 0)
    w = state["weights"][..., None]
    if not case["backward"]:
        return (_taken(state) * w).sum(1).to(state["z"].dtype)
    d, s = state["dout"].float()[:, None], state["slots"].long().flatten()
    dw = (_taken(state) * d).sum(-1)
    z = state["z"]
    dz = torch.zeros((z.shape[0] + 1, z.shape[1]), dtype=z.dtype, device=z.device)
    dz[torch.where(s >= 0, s, z.shape[0])] = (w * d).to(z.dtype).flatten(0, 1)
    return dz[:-1], dw


# ---- one pass

def run(state):
    if not own:
        return _plain(state)
    import paper_2608_26581_amd as rfq
    case = state["case"]
    op = case["op"]
    if op == "route":
        if case["backward"]:
            return rfq.rfq_route_backward(state["dweights"], state["logits"], state["weights"],
                                          state["experts"], renormalize=case["renormalize"])
        return rfq.rfq_route(state["logits"], case["k"], renormalize=case["renormalize"])
    if op == "sort":
        return tuple(rfq.rfq_expert_sort(state["experts"], case["E"], first=case["first"]))
    if op == "product":
        return rfq.rfq_gemm_experts(*state["a"], *state["w"], state["offsets"],
                                    rows=state["rows"] if case["mapped"] else None, out=state["z"])
    plan = state["offsets"], state["rows"], state["slots"]
    if op == "gather":
        return rfq.rfq_expert_gather(state["x"], plan)
    if case["backward"]:
        return rfq.rfq_expert_combine_backward(state["dout"], state["z"], state["weights"], plan)
    return rfq.rfq_expert_combine(state["z"], state["weights"], plan)


# ---- what a pass cannot do without

def work(case):
    op, T, k = case["op"], case["T"], case["k"]
    P = T * k
    size = {"bf16": 2, "f32": 4}
    if op == "route":
        logits = T * case["all"] * size[case["x"]]
        if case["backward"]:
            return {"bytes": (logits if case["renormalize"] else 2 * logits) + 12 * P,
                    "flops": 5 * T * case["all"]}
        return {"bytes": logits + 8 * P, "flops": 4 * T * case["all"]}
    if op == "sort":
        return {"bytes": 12 * P + 4 * case["E"], "flops": 0}
    # The pairs of this device's experts, all experts being as likely.
    held = P * case["E"] / case["all"]
    if op == "product":
        K, N, E = case["K"], case["N"], case["E"]
        parts, mx = 1 + case["residual"], 17 / 32
        M = min(T, held) if case["mapped"] else held
        chosen = E * (1 - (1 - k / case["all"]) ** T)
        return {"bytes": parts * M * K * mx + chosen * N * K * mx + held * N * size[case["z"]]
                + 4 * held * case["mapped"] + 4 * E, "flops": 2 * parts * held * N * K}
    row = case["N"] * size[case["x"]]
    if op == "gather":
        return {"bytes": min(T, held) * row + P * row + 4 * P, "flops": 0}
    if case["backward"]:
        return {"bytes": T * row + held * row + P * row + 12 * P, "flops": 3 * held * case["N"]}
    return {"bytes": held * row + T * row + 8 * P, "flops": 2 * held * case["N"]}


# ---- the same values in 64 bits

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


def _exact_route(case, state):
    l = state["logits"].double()
    T, E = l.shape
    at = torch.arange(E, device=l.device)
    left, values, mine = l.clone(), [], []
    for _ in range(case["k"]):
        top = left.amax(1)
        first = torch.where(left == top[:, None], at, E - 1).amin(1)
        values.append(torch.where(top == -math.inf, -math.inf, top))
        mine.append(torch.where(top == -math.inf, E, first))
        left[torch.arange(T, device=l.device), first] = -math.inf
    v, mine = torch.stack(values, 1), torch.stack(mine, 1)
    over = torch.logsumexp(v if case["renormalize"] else l, 1, keepdim=True)
    live = over > -math.inf
    return torch.where(live, torch.exp(v - torch.where(live, over, 0.0)), 0.0), mine, over


def exact(case, seed):
    op = case["op"]
    if op == "sort":
        return None                                     # whole numbers
    state = prepare(case, seed)
    if op == "route":
        w, mine, over = _exact_route(case, state)
        if not case["backward"]:
            return w, None
        # As the gradient is defined at the weights that the pass is given.
        l, d = state["logits"].double(), state["dweights"].double()
        w = state["weights"].double()
        chosen = torch.zeros((l.shape[0], l.shape[1] + 1), dtype=torch.float64, device=l.device)
        chosen.scatter_(1, mine, w * d)
        chosen = chosen[:, :-1]
        if case["renormalize"]:
            share = torch.zeros((l.shape[0], l.shape[1] + 1), dtype=torch.float64, device=l.device)
            share = share.scatter_(1, mine, w)[:, :-1]
        else:
            share = torch.where(over > -math.inf, torch.exp(l - over), 0.0)
        return chosen - share * (w * d).sum(1, keepdim=True)
    if op == "product":
        z = torch.zeros_like(state["z"], dtype=torch.float64)
        x = _values(*state["a"][:2])
        if case["residual"]:
            x = x + _values(*state["a"][2:])
        ends = state["offsets"].tolist()
        for e, (i, j) in enumerate(zip(ends, ends[1:])):
            if i < j:
                own_rows = x[state["rows"][i:j].long()] if case["mapped"] else x[i:j]
                z[i:j] = own_rows @ _values(state["w"][0][e], state["w"][1][e]).T.contiguous()
        return z
    if op == "gather":
        x = state["x"].double()
        return torch.cat((x, torch.zeros_like(x[:1])))[state["rows"].long()]
    z, slots = state["z"].double(), state["slots"].long()
    w = state["weights"].double()
    if not case["backward"]:
        out = torch.zeros((case["T"], case["N"]), dtype=torch.float64, device=z.device)
        for j in range(case["k"]):
            t = torch.nonzero(slots[:, j] >= 0).flatten()
            out[t] += w[t, j, None] * z[slots[t, j]]
        return out
    d = state["dout"].double()
    dz, dw = torch.zeros_like(z), torch.zeros_like(w)
    for j in range(case["k"]):
        t = torch.nonzero(slots[:, j] >= 0).flatten()
        dz[slots[t, j]] = w[t, j, None] * d[t]
        dw[t, j] = torch.linalg.vecdot(z[slots[t, j]], d[t])
    return dz, dw
