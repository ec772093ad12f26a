"""The 4-bit operators and the balance loss of include/tuna_moe.h, written from their definitions in 64 bits on the CPU."""
import torch

from moe_plain import swiglu  # noqa: F401

BLOCK = 32
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def blocks(n, size=BLOCK):
    return -(-n // size)


def from_codes(codes):
    c = codes.long()
    return torch.where(c >= 8, -1.0, 1.0) * VALUES[c & 7]


def to_codes(v):
    """To nearest, ties to the even code; magnitudes up to 6."""
    mid = (VALUES[1:] + VALUES[:-1]) / 2
    a = v.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, m in enumerate(mid):
        code += (a > m) if i % 2 == 0 else (a >= m)              # between code i and i + 1
    return code + 8 * torch.signbit(v).to(torch.uint8)


def scale_bytes(peak):
    """The smallest power of two that is not below peak / 6, as a byte; exact: peak is a 32-bit value."""
    m, e = torch.frexp(peak)                                     # peak = m 2^e, 0.5 <= m < 1; peak / 6 = m / 0.75 * 2^(e - 3)
    s = torch.where(m <= 0.75, e - 3, e - 2) + 127
    return torch.where(peak == 0, 127, s.clamp_min(1)).to(torch.uint8)


def quantise(x):
    """(codes, scale bytes) of the last axis in blocks of 32."""
    n = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    fine = x.isfinite().all(-1)
    x = torch.where(fine[..., None], x, 0.0)
    s = scale_bytes(x.abs().amax(-1))
    codes = to_codes(x / torch.exp2(s.double() - 127)[..., None])
    codes = torch.where(fine[..., None], codes, 0).to(torch.uint8)
    return codes.flatten(-2)[..., :n], torch.where(fine, s, 255).to(torch.uint8)


def packed(codes):
    n = codes.shape[-1]
    codes = torch.nn.functional.pad(codes, (0, n % 2))
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpacked(q, n):
    return torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :n]


def power(s):
    return torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127))


def wide(codes, s):
    return from_codes(codes) * power(s).repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]


def held(x):
    return wide(*quantise(x))


def quantise_columns(x, rows, nb):
    """Codes [cols, 128 nb] and scale bytes [cols, 4 nb] of the groups' rows, each padded to 128; and how many blocks of 128 are written."""
    cols = x.shape[1]
    q, s, at = torch.zeros(cols, 128 * nb, dtype=torch.uint8), torch.zeros(cols, 4 * nb, dtype=torch.uint8), 0
    for a, b in zip(rows[:-1], rows[1:]):
        n = blocks(b - a, 128)
        if n:
            c, sc = quantise(torch.nn.functional.pad(x[a:b].t().double(), (0, n * 128 - (b - a))))
            q[:, at * 128:(at + n) * 128], s[:, at * 4:(at + n) * 4] = c, sc
        at += n
    return q, s, at


def softmax(logits):
    l = logits.double()
    l = torch.where(l.isnan(), -torch.inf, l)
    top = l.amax(-1, keepdim=True)
    share = torch.where(top == torch.inf, (l == torch.inf).double(), torch.exp(l - torch.where(top.isinf(), 0.0, top)))
    share = torch.where(l == -torch.inf, 0.0, share)
    return share / share.sum(-1, keepdim=True).clamp_min(1e-300)


def balance(logits, experts, rows):
    """(counts, tokens, shares, loss) of the sequences rows[s] .. rows[s + 1] - 1."""
    e, p = logits.shape[1], softmax(logits)
    counts, tokens, shares, loss = [], [], [], []
    for a, b in zip(rows[:-1], rows[1:]):
        ex = experts[a:b].reshape(-1).long()
        c = torch.bincount(ex[(ex >= 0) & (ex < e)], minlength=e)
        n = int((p[a:b].sum(-1) > 0).sum())
        m = p[a:b].sum(0) / max(n, 1)
        counts.append(c)
        tokens.append(n)
        shares.append(m)
        loss.append(e * (c * m).sum() / max(int(c.sum()), 1))
    return torch.stack(counts), torch.tensor(tokens), torch.stack(shares), torch.stack(loss)


def balance_grad(logits, counts, tokens, rows, dloss):
    e, p = logits.shape[1], softmax(logits)
    out = torch.zeros_like(p)
    for s, (a, b) in enumerate(zip(rows[:-1], rows[1:])):
        if tokens[s] and counts[s].sum():
            f = counts[s].double() / counts[s].sum()
            out[a:b] = float(dloss[s]) * e / int(tokens[s]) * p[a:b] * (f - (p[a:b] @ f)[:, None])
    return out
