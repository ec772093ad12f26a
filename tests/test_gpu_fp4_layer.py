"""The 4-bit operators and the balance loss together, as a program runs them: a layer through the all-to-all, a training step, graphs, streams, another thread's call."""
import os
import sys
import threading

import pytest
import torch

import fp4_plain as plain
import moe_plain
import paper_2411_02581_amd as tuna

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U8 = torch.uint8
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


@pytest.fixture(scope="module", autouse=True)
def memory_is_given_back():
    yield
    torch.cuda.empty_cache()


def ok(rc):
    assert rc == tuna.TUNA_OK, tuna.tuna_strerror(rc)


def up(n, to):
    return -(-n // to) * to


@pytest.mark.parametrize("tokens,hidden,inner,experts,k,per_node", [(90, 384, 144, 12, 3, 4), (50, 272, 96, 8, 2, 0), (5, 128, 48, 16, 4, 0), (70, 512, 512, 6, 2, 2)])
def test_a_layer_through_the_all_to_all(tokens, hidden, inner, experts, k, per_node):
    import expert_parallel
    layer, x, logits, out, step = expert_parallel.main(tokens, hidden, inner, experts, k, per_node, 4)
    x, logits = x.cpu(), logits.cpu()
    _, names, weights = moe_plain.route(logits, k, True)
    assert torch.equal(layer.chosen.cpu().long(), names)
    w1, w2 = (plain.wide(plain.unpacked(q.cpu(), n), s.cpu()) for q, s, n in ((layer.w1, layer.s1, hidden), (layer.w2, layer.s2, inner)))
    want = torch.zeros(tokens, hidden, dtype=torch.float64)
    xq = plain.held(x)
    for t in range(tokens):
        for j in range(k):
            e = int(names[t, j])
            h = plain.held(plain.swiglu((w1[e] @ xq[t]).bfloat16())[None])[0]
            want[t] += weights[t, j] * (w2[e] @ h).bfloat16().double()
    # the same roundings on both sides but where a value lies at a rounding's edge: a few in a thousand of the activations, by a step of bf16 (2^-8), and of
    # those a few in a hundred by a step of e2m1 (up to a third); and the last roundings
    assert (out.cpu().double() - want).norm() <= 0.02 * want.norm()
    exact, _ = moe_plain.few(x[:step.shape[0]], logits[:step.shape[0]], k, True, w1, w2)
    assert (step.cpu().double() - exact).norm() <= 2.0 ** -8 * exact.norm()
    loss, counts = layer.balance(logits.to(DEV), layer.chosen)
    c, _, _, l = plain.balance(logits, names, [0, tokens])
    assert torch.equal(counts.cpu().long(), c[0]) and abs(float(loss) - float(l[0])) <= 1e-5 * float(l[0])


def test_the_layer_refuses_other_widths():
    import expert_parallel
    with pytest.raises(ValueError):
        expert_parallel.ExpertParallel(torch.zeros(2, 4, 4), torch.zeros(2, 4, 2), 1, 4, bits=6)


class Step:
    """Buffers of a training step of one linear layer of each expert, in 4 bits, with the router's balance loss."""

    def __init__(self, m, n, k, bounds, seed):
        g, e = gen(seed), len(bounds) - 1
        self.m, self.n, self.k, self.e = m, n, k, e
        self.rows = torch.tensor(bounds, dtype=torch.int32, device=DEV)
        self.x, self.dy = (torch.randn(m, c, generator=g, device=DEV).bfloat16() for c in (k, n))
        self.w = torch.randn(e * n, k, generator=g, device=DEV)
        self.logits = torch.randn(m, e, generator=g, device=DEV)
        self.at = torch.arange(e + 1, dtype=torch.int32, device=DEV) * n
        self.dloss = torch.ones(1, device=DEV)
        self.new()

    def new(self):
        m, n, k, e = self.m, self.n, self.k, self.e
        b = lambda *s: torch.zeros(*s, dtype=U8, device=DEV)  # noqa: E731
        wide, per = up(m, 128) + (e - 1) * 128, up(n, 128)
        wn = up(e * n, 128) + (e - 1) * 128
        self.b = dict(wq=b(e * n, up(k, 32) // 2), ws=b(e * n, up(k // 32 + 1, 16)), tq=b(k, wn // 2), ts=b(k, up(wn // 32, 16)),
                      xq=b(m, up(k, 32) // 2), xs=b(m, up(k // 32 + 1, 16)), dq=b(m, up(n, 32) // 2), ds=b(m, up(n // 32 + 1, 16)),
                      xtq=b(k, wide // 2), xts=b(k, up(wide // 32, 16)), dtq=b(n, wide // 2), dts=b(n, up(wide // 32, 16)))
        f = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
        i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
        rc, size = tuna.tuna_moe_balance_workspace(m, e, 1)
        ok(rc)
        rc, more = tuna.tuna_moe_route_workspace(m, e, 1, False)
        ok(rc)
        self.ws, self.ws2 = torch.empty(max(size, 16), dtype=U8, device=DEV), torch.empty(max(more, 16), dtype=U8, device=DEV)
        self.out = dict(y=f(m, n), dx=f(m, k), dw=f(e, n, k), counts=i(1, e), tokens=i(1), shares=f(1, e), loss=f(1), dlogits=f(m, e), experts=i(m, 1), weights=f(m, 1),
                        slots=i(m, 1), expert_rows=i(e + 1))
        self.per = per

    def run(self, stream=None):
        b, o, m, n, k, e, ld = self.b, self.out, self.m, self.n, self.k, self.e, lambda v: v.stride(0)
        kw = {} if stream is None else {"stream": stream}
        ok(tuna.tuna_fp4_quantize(self.w, 0, k, e * n, k, 0, None, 1, e * n, b["wq"], ld(b["wq"]), b["ws"], ld(b["ws"]), **kw))
        ok(tuna.tuna_fp4_quantize_columns(self.w, 0, k, e * n, k, self.at, e, b["tq"], ld(b["tq"]), b["ts"], ld(b["ts"]), **kw))
        for v, c, q, s, tq, ts in ((self.x, k, "xq", "xs", "xtq", "xts"), (self.dy, n, "dq", "ds", "dtq", "dts")):
            ok(tuna.tuna_fp4_quantize(v, 1, c, m, c, 0, None, 1, m, b[q], ld(b[q]), b[s], ld(b[s]), **kw))
            ok(tuna.tuna_fp4_quantize_columns(v, 1, c, m, c, self.rows, e, b[tq], ld(b[tq]), b[ts], ld(b[ts]), **kw))
        ok(tuna.tuna_fp4_matmul(b["xq"], ld(b["xq"]), b["xs"], ld(b["xs"]), b["wq"], ld(b["wq"]), n * ld(b["wq"]), b["ws"], ld(b["ws"]), n * ld(b["ws"]), self.rows, e,
                                o["y"], 0, n, m, n, k, **kw))
        ok(tuna.tuna_fp4_matmul(b["dq"], ld(b["dq"]), b["ds"], ld(b["ds"]), b["tq"], ld(b["tq"]), self.per // 2, b["ts"], ld(b["ts"]), self.per // 32, self.rows, e,
                                o["dx"], 0, k, m, k, n, **kw))
        ok(tuna.tuna_fp4_matmul_grad_w(b["dtq"], ld(b["dtq"]), b["dts"], ld(b["dts"]), b["xtq"], ld(b["xtq"]), b["xts"], ld(b["xts"]), self.rows, e, o["dw"], 0, k, n * k,
                                       m, n, k, **kw))
        ok(tuna.tuna_moe_route(self.logits, 0, e, m, e, 1, 0, o["experts"], o["weights"], o["slots"], o["expert_rows"], 1, None, None, None, None, self.ws2, self.ws2.numel(), **kw))
        ok(tuna.tuna_moe_balance(self.logits, 0, e, m, e, o["experts"], 1, None, 1, o["counts"], o["tokens"], o["shares"], o["loss"], self.ws, self.ws.numel(), **kw))
        ok(tuna.tuna_moe_balance_grad(self.logits, 0, e, m, e, None, 1, o["counts"], o["tokens"], self.dloss, 0, o["dlogits"], e, **kw))

    def check(self):
        w = self.w.cpu().view(self.e, self.n, self.k)
        x, dy, o, r = self.x.cpu(), self.dy.cpu(), {n: v.cpu() for n, v in self.out.items()}, self.rows.tolist()
        xq, dq = plain.held(x), plain.held(dy)
        near = lambda got, a, b: (got.double() - a @ b).abs().le((a.shape[1] / 64 + 20) * 2.0 ** -23 * (a.abs() @ b.abs()) + 1e-30).all()  # noqa: E731
        for i in range(self.e):
            a, z = r[i], r[i + 1]
            if a < z:
                assert near(o["y"][a:z], xq[a:z], plain.held(w[i]).t()) and near(o["dx"][a:z], dq[a:z], plain.held(w[i].t()).t())
                assert near(o["dw"][i], plain.held(dy[a:z].t()), plain.held(x[a:z].t()).t())
            else:
                assert bool((o["dw"][i] == 0).all())
        c, t, s, l = plain.balance(self.logits.cpu(), o["experts"], [0, self.m])
        assert torch.equal(o["counts"].long(), c) and torch.allclose(o["loss"].double(), l, rtol=1e-5)
        d = plain.balance_grad(self.logits.cpu(), c, t, [0, self.m], torch.ones(1))
        assert torch.allclose(o["dlogits"].double(), d, rtol=1e-4, atol=1e-9)


SIZES = [(300, 150, 160, [0, 7, 7, 210, 300]), (1300, 1100, 1000, [0, 100, 700, 1300]), (37, 64, 96, [0, 37])]


@pytest.mark.parametrize("m,n,k,bounds", SIZES)
def test_a_training_step(m, n, k, bounds):
    s = Step(m, n, k, bounds, m)
    s.run()
    s.check()


@pytest.mark.parametrize("m,n,k,bounds", SIZES)
def test_a_training_step_in_a_graph_and_on_two_streams(m, n, k, bounds):
    eager, kept = Step(m, n, k, bounds, 1), Step(m, n, k, bounds, 1)
    eager.run()
    sides = [(torch.cuda.Stream(), Step(m, n, k, bounds, 1)) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, v in sides:
            with torch.cuda.stream(s):
                v.run()
    torch.cuda.synchronize()
    for _, v in sides:
        assert all(torch.equal(v.out[name], eager.out[name]) for name in v.out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=sides[0][0]):
        kept.run()
    for n_ in range(3):
        for v in (eager, kept):
            g = gen(50 + n_)
            v.x.copy_(torch.randn(m, k, generator=g, device=DEV).bfloat16())
            v.logits.copy_(torch.randn(m, v.e, generator=g, device=DEV))
        eager.run()
        for v in kept.out.values():
            v.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(kept.out[name], eager.out[name]) for name in kept.out)
    eager.check()


def test_calls_of_two_threads():
    """Two threads with streams and buffers of their own at once: no call keeps anything."""
    want = Step(300, 150, 160, [0, 7, 7, 210, 300], 1)
    want.run()
    torch.cuda.synchronize()
    mine = [Step(300, 150, 160, [0, 7, 7, 210, 300], 1) for _ in range(2)]
    streams, wrong = [torch.cuda.Stream() for _ in range(2)], []

    def work(i):
        try:
            for _ in range(10):
                mine[i].run(streams[i])
            streams[i].synchronize()
        except BaseException as e:  # noqa: BLE001
            wrong.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong
    for v in mine:
        assert all(torch.equal(v.out[name], want.out[name]) for name in v.out)


@pytest.mark.parametrize("t", [1, 3, 20, 60])
def test_the_layer_for_few_tokens_in_a_graph_and_beside_other_work(t):
    h, f, e, k = 1024, 640, 16, 4
    g = gen(1)
    rb = lambda *s: torch.randint(0, 256, s, generator=g, device=DEV, dtype=U8)  # noqa: E731
    w1, w2 = rb(e, 2 * f, h // 2), rb(e, h, f // 2)
    s1, s2 = (torch.randint(118, 122, s, generator=g, device=DEV, dtype=U8) for s in ((e, 2 * f, h // 32), (e, h, f // 32)))
    x, logits = torch.randn(t, h, generator=g, device=DEV).bfloat16(), torch.randn(t, e, generator=g, device=DEV)
    rc, size = tuna.tuna_moe_few_workspace(t, h, f, e, k)
    ok(rc)
    new = lambda: (torch.zeros(t, h, device=DEV), torch.zeros(size, dtype=U8, device=DEV))  # noqa: E731

    def step(out, ws):
        ok(tuna.tuna_moe_few(x, h, t, h, logits, 0, e, e, k, 1, w1, s1, w2, s2, f, tuna.TUNA_F4, tuna.TUNA_SCALE_E8, out, tuna.TUNA_F32, h, ws, size))

    eager, kept, sides = new(), new(), [(torch.cuda.Stream(), new()) for _ in range(2)]
    step(*eager)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, buf in sides:
            with torch.cuda.stream(s):
                step(*buf)
    torch.cuda.synchronize()
    for _, buf in sides:
        assert torch.equal(buf[0], eager[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=sides[0][0]):
        step(*kept)
    for n in range(3):
        x.copy_(torch.randn(t, h, generator=gen(10 + n), device=DEV).bfloat16())
        logits.copy_(torch.randn(t, e, generator=gen(20 + n), device=DEV))
        step(*eager)
        kept[0].fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept[0], eager[0])


@pytest.mark.parametrize("bits", [4, 8])
def test_many_tokens_of_one_expert_give_the_same_every_time(bits):
    """More pairs of an expert than one task has: which task a pair is in does not depend on the order in which threads come."""
    t, h, f, e, k = 64, 512, 640, 12, 4
    g = gen(1)
    d = 2 if bits == 4 else 1
    rb = lambda *s: torch.randint(0, 100, s, generator=g, device=DEV, dtype=U8)  # noqa: E731
    w1, w2 = rb(e, 2 * f, h // d), rb(e, h, f // d)
    shapes = ((e, 2 * f, h // 32), (e, h, f // 32)) if bits == 4 else ((e, 2 * f // 128, h // 128), (e, h // 128, f // 128))
    s1, s2 = (torch.full(s, 110, dtype=U8, device=DEV) for s in shapes)
    x, logits = torch.randn(t, h, generator=g, device=DEV).bfloat16(), torch.randn(t, e, generator=g, device=DEV)
    logits[:, :2] += 100
    rc, size = tuna.tuna_moe_few_workspace(t, h, f, e, k)
    ok(rc)
    ws, first = torch.zeros(size, dtype=U8, device=DEV), None
    for _ in range(40):
        out = torch.zeros(t, h, device=DEV)
        ok(tuna.tuna_moe_few(x, h, t, h, logits, 0, e, e, k, 1, w1, s1, w2, s2, f, tuna.TUNA_F4 if bits == 4 else tuna.TUNA_F8, tuna.TUNA_SCALE_E8, out, 0, h, ws, size))
        first = out if first is None else first
        assert torch.equal(out, first)


def test_few_tokens_with_weights_beyond_32_bits():
    experts, inner, hidden = 130, 4096, 8192                     # 32 MB + 16 MB of values an expert: 6.5 GB
    w1 = torch.zeros(experts, 2 * inner, hidden // 2, dtype=U8, device=DEV)
    w2 = torch.zeros(experts, hidden, inner // 2, dtype=U8, device=DEV)
    g = gen(1)
    w1[-1], w2[-1] = (torch.randint(0, 256, v.shape[1:], generator=g, device=DEV, dtype=U8) for v in (w1, w2))
    s1 = torch.full((experts, 2 * inner, hidden // 32), 117, dtype=U8, device=DEV)
    s2 = torch.full((experts, hidden, inner // 32), 117, dtype=U8, device=DEV)
    for t in (1, 2):
        x = torch.randn(t, hidden, generator=g, device=DEV).bfloat16()
        logits = torch.zeros(t, experts, device=DEV)
        logits[:, -1] = 1
        rc, size = tuna.tuna_moe_few_workspace(t, hidden, inner, experts, 1)
        ws, out = torch.zeros(size, dtype=U8, device=DEV), torch.zeros(t, hidden, device=DEV)
        ok(tuna.tuna_moe_few(x, hidden, t, hidden, logits, 0, experts, experts, 1, 1, w1, s1, w2, s2, inner, tuna.TUNA_F4, tuna.TUNA_SCALE_E8, out, 0, hidden, ws, size))
        v1, v2 = (plain.wide(plain.unpacked(w[-1].cpu(), n), s[-1].cpu()) for w, s, n in ((w1, s1, hidden), (w2, s2, inner)))
        a = plain.swiglu(x.cpu().double() @ v1.t())
        assert bool(((out.cpu().double() - a @ v2.t()).abs() <= 2.0 ** -13 * (a.abs() @ v2.abs().t())).all())
