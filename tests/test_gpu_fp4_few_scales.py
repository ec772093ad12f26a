"""tuna_moe_few with 4-bit weights whose scales lie at the ends of their range, NaN (255) and powers of two from 2^-127 on, where weights are subnormal in bf16; and with
many pairs of an expert."""
import pytest
import torch

import fp4_plain as plain
import moe_plain
import paper_2411_02581_amd as tuna

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U8 = torch.uint8
# one token; the waves share the columns; each wave has its own; 32 tokens at a time; rows that do not start on 16 bytes; ends inside a block
SIZES = [(1, 512, 256, 8, 2), (6, 512, 320, 8, 2), (48, 512, 640, 24, 4), (64, 256, 512, 12, 4), (64, 256, 512, 3, 2), (9, 200, 88, 8, 2), (33, 720, 352, 8, 2)]


def ok(rc):
    assert rc == tuna.TUNA_OK, tuna.tuna_strerror(rc)


class Layer:
    def __init__(self, t, h, f, e, k):
        self.t, self.h, self.f, self.e, self.k = t, h, f, e, k
        g = torch.Generator().manual_seed(t * h)
        self.x, self.logits = torch.randn(t, h, generator=g).bfloat16(), torch.randn(t, e, generator=g)
        self.q = [torch.randint(0, 16, s, generator=g, dtype=U8) for s in ((e, 2 * f, h), (e, h, f))]
        self.s = [torch.randint(118, 124, (e, r, plain.blocks(c)), generator=g, dtype=U8) for r, c in ((2 * f, h), (h, f))]
        _, self.names, _ = moe_plain.route(self.logits, k, True)

    def run(self):
        t, h, f, e, k = self.t, self.h, self.f, self.e, self.k
        rc, size = tuna.tuna_moe_few_workspace(t, h, f, e, k)
        ok(rc)
        ws, out = torch.zeros(size, dtype=U8, device=DEV), torch.zeros(t, h, device=DEV)
        w1, w2 = (plain.packed(q).contiguous().to(DEV) for q in self.q)
        s1, s2 = (s.to(DEV) for s in self.s)
        ok(tuna.tuna_moe_few(self.x.to(DEV), h, t, h, self.logits.to(DEV), 0, e, e, k, tuna.TUNA_ROUTE_RENORM, w1, s1, w2, s2, f, tuna.TUNA_F4, tuna.TUNA_SCALE_E8, out, 0, h,
                             ws, size))
        return out.cpu()

    def check(self):
        got = self.run()
        exact, size = moe_plain.few(self.x, self.logits, self.k, True, *(plain.wide(q, s) for q, s in zip(self.q, self.s)))
        assert float(size.min()) > 1e-30                         # (the result is no subnormal number)
        # as in test_gpu_fp4.py: the activations in two bf16 parts, 2^-16 of each, and sums in 32 bits
        assert bool(((got.double() - exact).abs() <= 2.0 ** -13 * size).all())


@pytest.mark.parametrize("t,h,f,e,k", SIZES)
@pytest.mark.parametrize("block", [0, -1])
def test_a_scale_that_is_not_a_number(t, h, f, e, k, block):
    """In a row of w1: all that the expert's tokens get; in a row of w2: its column of their results.  Other tokens do not see it."""
    layer = Layer(t, h, f, e, k)
    bad = int(layer.names[t // 2, 0])
    has = (layer.names == bad).any(1)
    layer.s[1][bad, h - 1, block] = 255
    got = layer.run().isnan()
    assert torch.equal(got[:, h - 1], has) and not bool(got[:, :h - 1].any())
    layer.s[0][bad, f // 2, block] = 255
    got = layer.run().isnan()
    assert torch.equal(got, has[:, None].expand(t, h))


@pytest.mark.parametrize("t,h,f,e,k", SIZES)
def test_weights_that_are_subnormal_in_bf16(t, h, f, e, k):
    """Scales of 2^-127 to 2^-122 in either product, beside tokens (or activations) that are as large as these are small."""
    layer = Layer(t, h, f, e, k)
    layer.s[0] -= 118                                            # 0 to 5
    layer.x = (layer.x.float() * 2.0 ** 118).bfloat16()
    layer.check()
    layer = Layer(t, h, f, e, k)
    layer.s[1] -= 118
    layer.x = (layer.x.float() * 2.0 ** 30).bfloat16()
    layer.check()


@pytest.mark.parametrize("t,h,f,e,k", SIZES)
def test_large_scales(t, h, f, e, k):
    """Up to 2^125, whose largest weight is 6 * 2^125: bf16 holds it."""
    layer = Layer(t, h, f, e, k)
    layer.s[0] += 2                                              # 120 to 125
    layer.s[0] = (layer.s[0].int() + 127).clamp_max(252).to(U8)
    layer.x = (layer.x.float() * 2.0 ** -125).bfloat16()
    layer.check()


@pytest.mark.parametrize("t,h,f,e,k", [(64, 200, 88, 2, 2), (64, 200, 88, 3, 2), (40, 1000, 232, 4, 4), (64, 200, 88, 20, 1), (64, 256, 512, 2, 2), (33, 512, 640, 3, 3)])
def test_more_pairs_of_an_expert_than_a_task_has(t, h, f, e, k):
    """Sixteen pairs, or four where rows start on 16 bytes: the same every time."""
    layer = Layer(t, h, f, e, k)
    layer.check()
    first = layer.run()
    for _ in range(5):
        assert torch.equal(layer.run(), first)
