"""The operators of include/tuna_moe.h from their definitions, in 64 bits on the CPU: what the tests compare with."""
import math

import torch

BLOCK = 128


def blocks(n):
    return -(-n // BLOCK)


# ------------------------------------------------------------------------------------------------ routing


def route(logits, k, renorm):
    """(softmax, experts, weights) of logits of any type; experts -1 and weight 0 where fewer than k are eligible."""
    l = logits.double().clone()
    l[l.isnan()] = -math.inf
    t, e = l.shape
    p = torch.zeros_like(l)
    experts = torch.full((t, k), -1, dtype=torch.int64)
    weights = torch.zeros(t, k, dtype=torch.float64)
    for i in range(t):
        there = [j for j in range(e) if l[i, j] > -math.inf]
        if not there:
            continue
        top = max(float(l[i, j]) for j in there)
        share = {j: (1.0 if l[i, j] == top else 0.0) if top == math.inf else math.exp(float(l[i, j]) - top) for j in there}
        total = sum(share.values())
        for j in there:
            p[i, j] = share[j] / total
        best = sorted(there, key=lambda j: (-float(l[i, j]), j))[:k]
        part = sum(share[j] for j in best) if renorm else total
        for n, j in enumerate(best):
            experts[i, n] = j
            weights[i, n] = share[j] / part
    return p, experts, weights


def places(experts, n_experts, plan, row_bytes=1):
    """(slots, expert_rows, sendcounts, sdispls, recvcounts, rdispls), the last four of records of row_bytes bytes."""
    t, k = experts.shape
    shard = -(-t // n_experts) if plan and t else max(t, 1)
    pairs = sorted((i // shard, int(experts[i, j]), i, j) for i in range(t) for j in range(k) if experts[i, j] >= 0)
    slots = torch.full((t, k), -1, dtype=torch.int64)
    send = torch.zeros(n_experts, n_experts, dtype=torch.int64)
    for at, (rank, e, i, j) in enumerate(pairs):
        slots[i, j] = at
        if plan:
            send[rank, e] += 1
    rows = torch.zeros(n_experts + 1, dtype=torch.int64)
    for _, e, _, _ in pairs:
        rows[e + 1] += 1
    prefix = lambda m: (torch.cumsum(m.reshape(-1), 0) - m.reshape(-1)).reshape(m.shape) * row_bytes  # noqa: E731
    recv = send.t().contiguous()
    return slots, torch.cumsum(rows, 0), send * row_bytes, prefix(send), recv * row_bytes, prefix(recv)


def route_grad(p, experts, weights, dweights, renorm):
    t, e = p.shape
    d = torch.zeros_like(p)
    for i in range(t):
        chosen = [(int(experts[i, j]), j) for j in range(experts.shape[1]) if experts[i, j] >= 0]
        s = sum(float(weights[i, j]) * float(dweights[i, j]) for _, j in chosen)
        g = {n: float(dweights[i, j]) for n, j in chosen}
        if renorm:
            for n, j in chosen:
                d[i, n] = float(weights[i, j]) * (g[n] - s)
        else:
            for n in range(e):
                d[i, n] = float(p[i, n]) * (g.get(n, 0.0) - s)
    return d


# ------------------------------------------------------------------------------------------------ 8 bits

# every finite e4m3 value that is not negative, in order: its code is its place
E4M3 = torch.tensor([(m / 8) * 2.0 ** -6 if x == 0 else (1 + m / 8) * 2.0 ** (x - 7) for x in range(16) for m in range(8)][:127], dtype=torch.float64)


def to_e4m3(v):
    """Codes of the nearest values, ties to the even code; values up to 464 in magnitude.  Not finite: 0x7f."""
    fine = v.isfinite()
    a = torch.where(fine, v.abs(), 0.0)
    hi = torch.searchsorted(E4M3, a).clamp_max(126)
    lo = (hi - 1).clamp_min(0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = torch.where(torch.signbit(v), code + 128, code)
    return torch.where(fine, code, 0x7F).to(torch.uint8)


def from_e4m3(code):
    c = code.long()
    v = torch.where((c & 127) == 127, math.nan, E4M3[(c & 127).clamp_max(126)])
    return torch.where(c >= 128, -v, v)


def scales(peak, kind):
    """(value, as stored) for the largest finite magnitudes of blocks, 64 bits."""
    s = (peak / 448).float().clamp_min(2.0 ** -126).double()     # rounded to 32 bits once: the quotient in 64 bits is far closer
    if kind == "e8":
        m, e = torch.frexp(s)
        e = torch.where(m == 0.5, e - 1, e)
        e = torch.where(peak == 0, 0, e)
        return torch.exp2(e.double()), (e + 127).to(torch.uint8)
    s = torch.where(peak == 0, 1.0, s)
    return s, s.float()


def quantise(x, kind):
    """(codes, scales as stored) by blocks of 128 along the last axis."""
    n = x.shape[-1]
    v = torch.nn.functional.pad(x.double(), (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    peak = torch.where(v.isfinite(), v.abs(), 0.0).amax(-1)
    s, stored = scales(peak, kind)
    q = v / s[..., None]
    if kind == "f32":
        q = torch.where(q.isfinite(), q.float().double(), q)     # the quotient is a 32-bit value
    return to_e4m3(q).flatten(-2)[..., :n].contiguous(), stored


def scale_values(s, kind):
    return torch.exp2(s.double() - 127) if kind == "e8" else s.double()


def wide(codes, s, kind, rows=1):
    s = scale_values(s, kind)
    i, j = torch.arange(codes.shape[-2]) // rows, torch.arange(codes.shape[-1]) // BLOCK
    return from_e4m3(codes) * s[..., i, :][..., j]


def quantise_columns(x, rows, kind, ldq):
    """Codes [cols, ldq] and stored scales [cols, ldq / 128] of the groups' rows, each padded to 128; and which columns are written."""
    cols = x.shape[1]
    q = torch.zeros(cols, ldq, dtype=torch.uint8)
    s = torch.zeros(cols, ldq // BLOCK, dtype=torch.uint8 if kind == "e8" else torch.float32)
    at = 0
    for a, b in zip(rows[:-1], rows[1:]):
        n = blocks(b - a)
        if n:
            part = torch.nn.functional.pad(x[a:b].t().double(), (0, n * BLOCK - (b - a)))
            c, sc = quantise(part, kind)
            q[:, at * BLOCK:(at + n) * BLOCK], s[:, at:at + n] = c, sc
        at += n
    return q, s, at


def silu(g):
    return g / (1 + torch.exp(-g))


def swiglu(x):
    g, u = x.double().chunk(2, -1)
    return silu(g) * u


def swiglu_grad(x, dh):
    g, u = x.double().chunk(2, -1)
    s = 1 / (1 + torch.exp(-g))
    d = dh.double()
    return torch.cat([d * u * s * (1 + g * (1 - s)), d * g * s], -1)


# ------------------------------------------------------------------------------------------------ sums


def combine(y, slots, weights):
    out = torch.zeros(slots.shape[0], y.shape[1], dtype=torch.float64)
    for t in range(slots.shape[0]):
        for j in range(slots.shape[1]):
            r = int(slots[t, j])
            if 0 <= r < y.shape[0]:
                out[t] += float(weights[t, j]) * y[r].double()
    return out


def few(x, logits, k, renorm, w1, w2):
    """w1 [experts, 2 inner, hidden], w2 [experts, hidden, inner] in 64 bits."""
    _, experts, weights = route(logits, k, renorm)
    out = torch.zeros(x.shape[0], w2.shape[1], dtype=torch.float64)
    size = torch.zeros_like(out)                                 # the sum of the magnitudes that are added
    for t in range(x.shape[0]):
        for j in range(k):
            e = int(experts[t, j])
            if e >= 0:
                h = swiglu(w1[e] @ x[t].double())
                out[t] += weights[t, j] * (w2[e] @ h)
                size[t] += weights[t, j] * (w2[e].abs() @ h.abs())
    return out, size
