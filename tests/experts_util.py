"""Plain 64-bit implementations of the calls around a layer of experts, on the CPU and
from their definitions, and inputs for the tests."""
import math

import torch


def route(logits, k, renormalize):
    """(weights [T][k], experts [T][k], spread [T]): per row, one choice after the other;
    spread: the largest distance of a chosen or (not renormalized) any logit from the largest."""
    rows = logits.double().cpu().tolist()
    W, X, S = [], [], []
    for row in rows:
        left = list(enumerate(row))
        chosen = []
        for _ in range(k):
            best = None
            for i, v in left:
                if v == -math.inf:
                    continue
                if best is None or (math.isnan(v) and not math.isnan(best[1])) or v > best[1]:
                    best = (i, v)
            if best is None:
                break
            chosen.append(best)
            left = [p for p in left if p[0] != best[0]]
        over = [v for _, v in chosen] if renormalize else [v for v in row if v != -math.inf]
        bad = any(math.isnan(v) or v == math.inf for v in over)
        m = max(over) if over and not bad else 0.0
        total = sum(math.exp(v - m) for v in over) if not bad else math.nan
        w = [math.nan if bad else math.exp(v - m) / total for _, v in chosen]
        W.append(w + [0.0] * (k - len(w)))
        X.append([i for i, _ in chosen] + [-1] * (k - len(chosen)))
        S.append(m - min(over) if over and not bad else 0.0)
    return torch.tensor(W, dtype=torch.float64), torch.tensor(X), torch.tensor(S, dtype=torch.float64)


def sort(experts, E, first=0):
    """(offsets, rows, slots) by going through the pairs of one expert after the other."""
    T, k = experts.shape
    pairs = experts.cpu().flatten().tolist()
    offsets, rows, slots = [0], [], [-1] * (T * k)
    for e in range(E):
        for p, x in enumerate(pairs):
            if x == first + e:
                slots[p] = len(rows)
                rows.append(p // k)
        offsets.append(len(rows))
    rows += [-1] * (T * k - len(rows))
    return (torch.tensor(offsets), torch.tensor(rows, dtype=torch.int64),
            torch.tensor(slots, dtype=torch.int64).reshape(T, k))


def choices(T, E, k, seed, skew=0.5):
    """int32 [T][k] different experts per token, some more popular than others."""
    g = torch.Generator().manual_seed(seed)
    l = torch.randn((T, E), generator=g) + skew * torch.randn((E,), generator=g)
    return torch.topk(l, k, dim=1).indices.int()


def plan_tensors(plan):
    return tuple(t.int().cuda() for t in plan)


_E2M1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6],
                     dtype=torch.float64)


def decode(codes, scales):
    """float64 values of MXFP4 codes (any leading sizes), NaN where the scale byte is 0xFF."""
    c, s = codes.cpu(), scales.cpu()
    v = _E2M1[torch.stack((c & 15, c >> 4), -1).flatten(-2).long()]
    f = torch.exp2(s.double() - 127)
    f[s == 255] = math.nan
    return v * f.repeat_interleave(32, -1)


def product(a, w, offsets, rows, M):
    """(Z [P][N], bound [P][N], live [P]) in 64 bits; live: the rows that belong to an expert."""
    x = decode(a[0], a[1])
    r = decode(a[2], a[3]) if a[2] is not None else torch.zeros_like(x)
    wv = decode(*w)
    E, N, K = wv.shape
    off = offsets.cpu().tolist()
    P = M if rows is None else rows.numel()
    z, bound = torch.zeros((P, N), dtype=torch.float64), torch.zeros((P, N), dtype=torch.float64)
    live = torch.zeros(P, dtype=torch.bool)
    at = torch.arange(P) if rows is None else rows.cpu().long()
    for e in range(E):
        i = min(max(off[e], 0), P)
        j = min(max(off[e + 1], i), P)
        if i == j:
            continue
        n = at[i:j]
        ok = ((n >= 0) & (n < M)).double()[:, None]
        n = n.clamp(0, max(M - 1, 0))
        if M:
            z[i:j] = (x[n] * ok + r[n] * ok) @ wv[e].T
            bound[i:j] = ((x[n].abs() + r[n].abs()) * ok) @ wv[e].abs().T
        live[i:j] = True
    return z, bound, live


def codes(rows, K, seed, residual=True, spread=3):
    """Random codes with scale bytes near 127 - spread .. 127 + spread."""
    g = torch.Generator().manual_seed(seed)

    def part(shape, lo, hi):
        return torch.randint(lo, hi, shape, generator=g, dtype=torch.uint8).cuda()
    q = part((*rows, K // 2), 0, 256), part((*rows, K // 32), 127 - spread, 128 + spread)
    if residual is None:
        return q
    r = (part((*rows, K // 2), 0, 256), part((*rows, K // 32), 124 - spread, 125 + spread))
    return (*q, *(r if residual else (None, None)))
