"""A mixture of experts whose rows travel through the all-to-all: one virtual rank per expert, the tokens cut into as many shards.

    python examples/expert_parallel.py [tokens hidden inner experts k experts_per_node]

Route, pack rows as 8-bit records, exchange, the experts' two products, exchange back, sum.  For a few tokens `ExpertParallel.step`
runs the whole layer in two kernels instead; both are compared when the file is run."""
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


class ExpertParallel:
    """w1 [experts, 2 inner, hidden] (gate rows, then up rows), w2 [experts, hidden, inner]; buffers for up to max_tokens tokens."""

    def __init__(self, w1, w2, k, max_tokens, experts_per_node=0):
        self.experts, self.hidden, self.inner = w2.shape
        self.k, self.per_node, self.max_tokens, dev = k, experts_per_node, max_tokens, w1.device
        (self.w1, self.s1), (self.w2, self.s2) = quantise_weights(w1), quantise_weights(w2)
        e, h, f, pairs = self.experts, self.hidden, self.inner, max_tokens * k
        self.record = -(-(h + _blocks(h)) // 16) * 16            # values, then scales; rows on 16 bytes
        new = lambda *s, dtype=torch.uint8: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.rows = new(e + 1, dtype=torch.int32)
        self.plan = [new(e, e, dtype=d) for d in (torch.int32, torch.int64) * 2]
        rc, size = tuna.tuna_moe_route_workspace(max_tokens, e, k, True)
        _ok(rc)
        rc, few = tuna.tuna_moe_few_workspace(min(max_tokens, tuna.TUNA_MOE_FEW_TOKENS), h, f, e, k)
        _ok(rc)
        self.workspace = new(max(size, few))
        self.send, self.recv = new(pairs, self.record), new(pairs, self.record)
        self.mid, self.q, self.qs = new(pairs, 2 * f, dtype=torch.bfloat16), new(pairs, f), new(pairs, _blocks(f))
        self.y, self.back = new(pairs, h, dtype=torch.bfloat16), new(pairs, h, dtype=torch.bfloat16)

    def _check(self, x, logits, most):
        """The buffers have room for `most` tokens, and the calls name the distances of dense rows."""
        t = x.shape[0]
        if t > most or x.shape != (t, self.hidden) or logits.shape != (t, self.experts):
            raise ValueError("up to %d tokens of %d columns and as many rows of %d logits expected" % (most, self.hidden, self.experts))
        if x.dtype != torch.bfloat16 or logits.dtype != torch.float32 or not x.is_contiguous() or not logits.is_contiguous():
            raise ValueError("contiguous bf16 tokens and 32-bit logits expected")

    def __call__(self, x, logits):
        self._check(x, logits, self.max_tokens)
        t, e, h, f, k = x.shape[0], self.experts, self.hidden, self.inner, self.k
        experts, slots = (torch.empty(t, k, dtype=torch.int32, device=x.device) for _ in range(2))
        weights, out, pairs = torch.empty(t, k, device=x.device), torch.empty_like(x), t * k
        _ok(tuna.tuna_moe_route(logits, tuna.TUNA_F32, e, t, e, k, tuna.TUNA_ROUTE_RENORM, experts, weights, slots, self.rows, 1, *self.plan,
                                self.workspace, self.workspace.numel()))
        send, recv = self.send[:pairs], self.recv[:pairs]
        _ok(tuna.tuna_fp8_quantize(x, tuna.TUNA_BF16, h, t, h, tuna.TUNA_ACT_NONE, slots, k, pairs, send, self.record, send[:, h:], self.record,
                                   tuna.TUNA_SCALE_E8))
        # the plan counts rows (records of one byte): times a record's size it is the call's
        sc, sd, rc, rd = (m * self.record for m in self.plan)
        _ok(tuna.tuna_alltoallv(send, sc, sd, recv, rc, rd, e, tuna.TUNA_RADIX_AUTO, self.per_node))
        nh, nf = _blocks(h), _blocks(f)
        _ok(tuna.tuna_fp8_matmul(recv, self.record, recv[:, h:], self.record, self.w1, h, 2 * f * h, self.s1, nh, self.s1[0].numel(), tuna.TUNA_SCALE_E8,
                                 self.rows, e, self.mid, tuna.TUNA_BF16, 2 * f, pairs, 2 * f, h))
        _ok(tuna.tuna_fp8_quantize(self.mid, tuna.TUNA_BF16, 2 * f, pairs, f, tuna.TUNA_ACT_SWIGLU, None, 1, pairs, self.q, f, self.qs, nf, tuna.TUNA_SCALE_E8))
        _ok(tuna.tuna_fp8_matmul(self.q, f, self.qs, nf, self.w2, f, h * f, self.s2, nf, self.s2[0].numel(), tuna.TUNA_SCALE_E8,
                                 self.rows, e, self.y, tuna.TUNA_BF16, h, pairs, h, f))
        sc, sd, rc, rd = (m * (2 * h) for m in self.plan)
        _ok(tuna.tuna_alltoallv(self.y, rc, rd, self.back, sc, sd, e, tuna.TUNA_RADIX_AUTO, self.per_node))
        _ok(tuna.tuna_moe_combine(self.back, tuna.TUNA_BF16, h, pairs, slots, weights, t, k, h, out, tuna.TUNA_BF16, h))
        return out

    def step(self, x, logits):
        self._check(x, logits, min(self.max_tokens, tuna.TUNA_MOE_FEW_TOKENS))
        t, e, h = x.shape[0], self.experts, self.hidden
        out = torch.empty_like(x)
        _ok(tuna.tuna_moe_few(x, h, t, h, logits, tuna.TUNA_F32, e, e, self.k, tuna.TUNA_ROUTE_RENORM, self.w1, self.s1, self.w2, self.s2, self.inner,
                              tuna.TUNA_F8, tuna.TUNA_SCALE_E8, out, tuna.TUNA_BF16, h, self.workspace, self.workspace.numel()))
        return out


def main(tokens=2000, hidden=1024, inner=512, experts=64, k=4, per_node=16):
    dev = "cuda:0"
    torch.manual_seed(0)
    w1 = torch.randn(experts, 2 * inner, hidden, device=dev) / hidden ** 0.5
    w2 = torch.randn(experts, hidden, inner, device=dev) / inner ** 0.5
    layer = ExpertParallel(w1, w2, k, tokens, per_node)
    x, logits = torch.randn(tokens, hidden, device=dev, dtype=torch.bfloat16), torch.randn(tokens, experts, device=dev)
    out = layer(x, logits)
    n = min(tokens, tuna.TUNA_MOE_FEW_TOKENS)
    few = layer.step(x[:n], logits[:n])
    off = (out[:n].float() - few.float()).norm() / few.float().norm()
    print("%d tokens through %d experts; %d of them in two kernels: the two differ by %.2g (rows in 8 bits on the first way)" % (tokens, experts, n, off))
    return layer, x, logits, out, few


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
