"""A mixture of experts whose rows travel through the all-to-all: one virtual rank per expert, the tokens cut into as many shards.

    python examples/expert_parallel.py [tokens hidden inner experts k experts_per_node bits]

Route, pack rows as records of 8-bit (or 4-bit) values, exchange, the experts' two products, exchange back, sum.  For a few tokens `ExpertParallel.step`
runs the whole layer in two kernels instead; both are compared when the file is run.  `ExpertParallel.balance` says how evenly the experts are used."""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch

import paper_2411_02581_amd as tuna

BLOCK = 128


def _ok(rc):
    if rc != tuna.TUNA_OK:
        raise RuntimeError(tuna.tuna_strerror(rc))


def _blocks(n):
    return -(-n // BLOCK)


def quantise_weights(w):
    """[experts, rows, cols] -> e4m3 values and a power-of-two scale (its exponent byte) for each 128 x 128 of them."""
    e, r, c = w.shape
    v = torch.nn.functional.pad(w.float(), (0, -c % BLOCK, 0, -r % BLOCK)).view(e, _blocks(r), BLOCK, _blocks(c), BLOCK)
    peak = v.abs().amax((2, 4))
    power = torch.where(peak > 0, torch.ceil(torch.log2(peak / 448)), 0.0)
    q = (v / torch.exp2(power)[:, :, None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return q.reshape(e, _blocks(r) * BLOCK, -1)[:, :r, :c].contiguous(), (power + 127).to(torch.uint8)


def quantise_weights_4(w):
    """[experts, rows, cols] -> e2m1 values, two to a byte, and a power-of-two scale (its exponent byte) for 32 neighbours of a row, rows back to back."""
    e, r, c = w.shape
    w = w.float().reshape(e * r, c).contiguous()
    q = torch.empty(e, r, -(-c // 2), dtype=torch.uint8, device=w.device)
    s = torch.empty(e, r, -(-c // 32), dtype=torch.uint8, device=w.device)
    _ok(tuna.tuna_fp4_quantize(w, tuna.TUNA_F32, c, e * r, c, tuna.TUNA_ACT_NONE, None, 1, e * r, q, q.shape[2], s, s.shape[2]))
    return q, s


def rows_on_16(s):
    """A copy of rows of scales in 4 bits that start on 16 bytes, as the products of many rows want them (tuna_moe_few takes them back to back)."""
    p = torch.zeros(*s.shape[:2], -(-s.shape[2] // 16) * 16, dtype=s.dtype, device=s.device)
    p[..., :s.shape[2]] = s
    return p


class ExpertParallel:
    """w1 [experts, 2 inner, hidden] (gate rows, then up rows), w2 [experts, hidden, inner]; buffers for up to max_tokens tokens; rows and weights in
    `bits` bits, 8 or 4."""

    def __init__(self, w1, w2, k, max_tokens, experts_per_node=0, bits=8):
        if bits not in (4, 8):
            raise ValueError("8 or 4 bits expected")
        self.experts, self.hidden, self.inner = w2.shape
        self.k, self.per_node, self.max_tokens, self.bits, dev = k, experts_per_node, max_tokens, bits, w1.device
        held = quantise_weights if bits == 8 else quantise_weights_4
        (self.w1, self.s1), (self.w2, self.s2) = held(w1), held(w2)
        self.p1, self.p2 = (self.s1, self.s2) if bits == 8 else (rows_on_16(self.s1), rows_on_16(self.s2))
        e, h, f, pairs = self.experts, self.hidden, self.inner, max_tokens * k
        size = (lambda n: (n, _blocks(n))) if bits == 8 else (lambda n: (-(-n // 2), -(-n // 32)))
        (self.h_bytes, h_scales), (self.f_bytes, f_scales) = size(h), size(f)       # of a row's values, and its scales
        self.f_scales = f_scales if bits == 8 else -(-f_scales // 16) * 16          # the distance of two rows'
        self.record = -(-(self.h_bytes + h_scales) // 16) * 16   # values, then scales; rows on 16 bytes
        new = lambda *s, dtype=torch.uint8: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.rows = new(e + 1, dtype=torch.int32)
        self.plan = [new(e, e, dtype=d) for d in (torch.int32, torch.int64) * 2]
        rc, size = tuna.tuna_moe_route_workspace(max_tokens, e, k, True)
        _ok(rc)
        rc, few = tuna.tuna_moe_few_workspace(min(max_tokens, tuna.TUNA_MOE_FEW_TOKENS), h, f, e, k)
        _ok(rc)
        self.workspace = new(max(size, few))
        self.send, self.recv = new(pairs, self.record), new(pairs, self.record)
        self.mid, self.q, self.qs = new(pairs, 2 * f, dtype=torch.bfloat16), new(pairs, self.f_bytes), new(pairs, self.f_scales)
        self.y, self.back = new(pairs, h, dtype=torch.bfloat16), new(pairs, h, dtype=torch.bfloat16)

    def _check(self, x, logits, most):
        """The buffers have room for `most` tokens, and the calls name the distances of dense rows."""
        t = x.shape[0]
        if t > most or x.shape != (t, self.hidden) or logits.shape != (t, self.experts):
            raise ValueError("up to %d tokens of %d columns and as many rows of %d logits expected" % (most, self.hidden, self.experts))
        if x.dtype != torch.bfloat16 or logits.dtype != torch.float32 or not x.is_contiguous() or not logits.is_contiguous():
            raise ValueError("contiguous bf16 tokens and 32-bit logits expected")

    def _pack(self, x, ldx, rows, cols, act, slots, copies, out_rows, q, ldq, scales, ld_scales):
        if self.bits == 8:
            _ok(tuna.tuna_fp8_quantize(x, tuna.TUNA_BF16, ldx, rows, cols, act, slots, copies, out_rows, q, ldq, scales, ld_scales, tuna.TUNA_SCALE_E8))
        else:
            _ok(tuna.tuna_fp4_quantize(x, tuna.TUNA_BF16, ldx, rows, cols, act, slots, copies, out_rows, q, ldq, scales, ld_scales))

    def _multiply(self, x, ldx, xs, ld_xs, w, s, y, m, n, k):
        """The rows of every expert times its weights, which lie back to back."""
        ldw, ld_ws, e = w.stride(1), s.stride(1), self.experts
        if self.bits == 8:
            _ok(tuna.tuna_fp8_matmul(x, ldx, xs, ld_xs, w, ldw, w.stride(0), s, ld_ws, s.stride(0), tuna.TUNA_SCALE_E8, self.rows, e, y, tuna.TUNA_BF16, n, m, n, k))
        else:
            _ok(tuna.tuna_fp4_matmul(x, ldx, xs, ld_xs, w, ldw, w.stride(0), s, ld_ws, s.stride(0), self.rows, e, y, tuna.TUNA_BF16, n, m, n, k))

    def balance(self, logits, experts):
        """(loss, pairs of every expert) of a batch: 1 where all experts are used evenly."""
        t, e = logits.shape
        if logits.dtype != torch.float32 or not logits.is_contiguous() or experts.shape != (t, self.k) or e != self.experts:
            raise ValueError("contiguous 32-bit logits and the router's choice expected")
        rc, size = tuna.tuna_moe_balance_workspace(t, e, 1)
        _ok(rc)
        new = lambda *s, dtype: torch.empty(*s, dtype=dtype, device=logits.device)  # noqa: E731
        counts, tokens, shares, loss, ws = new(1, e, dtype=torch.int32), new(1, dtype=torch.int32), new(1, e, dtype=torch.float32), new(1, dtype=torch.float32), \
            new(max(size, 16), dtype=torch.uint8)
        _ok(tuna.tuna_moe_balance(logits, tuna.TUNA_F32, e, t, e, experts, self.k, None, 1, counts, tokens, shares, loss, ws, ws.numel()))
        return loss[0], counts[0]

    def __call__(self, x, logits):
        self._check(x, logits, self.max_tokens)
        t, e, h, f, k = x.shape[0], self.experts, self.hidden, self.inner, self.k
        experts, slots = (torch.empty(t, k, dtype=torch.int32, device=x.device) for _ in range(2))
        weights, out, pairs = torch.empty(t, k, device=x.device), torch.empty_like(x), t * k
        _ok(tuna.tuna_moe_route(logits, tuna.TUNA_F32, e, t, e, k, tuna.TUNA_ROUTE_RENORM, experts, weights, slots, self.rows, 1, *self.plan,
                                self.workspace, self.workspace.numel()))
        self.chosen = experts
        send, recv = self.send[:pairs], self.recv[:pairs]
        self._pack(x, h, t, h, tuna.TUNA_ACT_NONE, slots, k, pairs, send, self.record, send[:, self.h_bytes:], self.record)
        # the plan counts rows (records of one byte): times a record's size it is the call's
        sc, sd, rc, rd = (m * self.record for m in self.plan)
        _ok(tuna.tuna_alltoallv(send, sc, sd, recv, rc, rd, e, tuna.TUNA_RADIX_AUTO, self.per_node))
        self._multiply(recv, self.record, recv[:, self.h_bytes:], self.record, self.w1, self.p1, self.mid, pairs, 2 * f, h)
        self._pack(self.mid, 2 * f, pairs, f, tuna.TUNA_ACT_SWIGLU, None, 1, pairs, self.q, self.f_bytes, self.qs, self.f_scales)
        self._multiply(self.q, self.f_bytes, self.qs, self.f_scales, self.w2, self.p2, self.y, pairs, h, f)
        sc, sd, rc, rd = (m * (2 * h) for m in self.plan)
        _ok(tuna.tuna_alltoallv(self.y, rc, rd, self.back, sc, sd, e, tuna.TUNA_RADIX_AUTO, self.per_node))
        _ok(tuna.tuna_moe_combine(self.back, tuna.TUNA_BF16, h, pairs, slots, weights, t, k, h, out, tuna.TUNA_BF16, h))
        return out

    def step(self, x, logits):
        self._check(x, logits, min(self.max_tokens, tuna.TUNA_MOE_FEW_TOKENS))
        t, e, h = x.shape[0], self.experts, self.hidden
        out = torch.empty_like(x)
        _ok(tuna.tuna_moe_few(x, h, t, h, logits, tuna.TUNA_F32, e, e, self.k, tuna.TUNA_ROUTE_RENORM, self.w1, self.s1, self.w2, self.s2, self.inner,
                              tuna.TUNA_F8 if self.bits == 8 else tuna.TUNA_F4, tuna.TUNA_SCALE_E8, out, tuna.TUNA_BF16, h, self.workspace, self.workspace.numel()))
        return out


def main(tokens=2000, hidden=1024, inner=512, experts=64, k=4, per_node=16, bits=8):
    dev = "cuda:0"
    torch.manual_seed(0)
    w1 = torch.randn(experts, 2 * inner, hidden, device=dev) / hidden ** 0.5
    w2 = torch.randn(experts, hidden, inner, device=dev) / inner ** 0.5
    layer = ExpertParallel(w1, w2, k, tokens, per_node, bits)
    x, logits = torch.randn(tokens, hidden, device=dev, dtype=torch.bfloat16), torch.randn(tokens, experts, device=dev)
    out = layer(x, logits)
    n = min(tokens, tuna.TUNA_MOE_FEW_TOKENS)
    few = layer.step(x[:n], logits[:n])
    off = (out[:n].float() - few.float()).norm() / few.float().norm()
    print("%d tokens through %d experts; %d of them in two kernels: the two differ by %.2g (rows in %d bits on the first way)" % (tokens, experts, n, off, bits))
    loss, counts = layer.balance(logits, layer.chosen)
    print("balance loss %.3f (1: even), %d to %d pairs an expert" % (float(loss), int(counts.min()), int(counts.max())))
    return layer, x, logits, out, few


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
