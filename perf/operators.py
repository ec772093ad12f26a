"""The operators that a mixture of experts needs around the all-to-all, from a single token to a training step.

The rows of a mixture of experts travel through `tuna_alltoallv`: rank = expert, the tokens are cut into as many shards.
Around it stand the router that makes the call's arrays, the packing of rows into 8-bit records, the experts' products,
the weighted sum of what comes back, and the whole layer for a few tokens.

Fields of a case
  op        route, quantise, matmul, combine or few
  tokens, hidden, experts, k     rows, columns, experts and chosen experts a token, where the operator has them
  train     the gradients belong to the pass
  scale     type of the scales of 128 values: "f32" or "e8" (a power of two in 8 bits)
Further ones are explained at the `prepare_*` that reads them.  Everywhere `ld` is the distance of rows in elements.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
BLOCK = 128
FLOAT8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one step of a server that generates for two dozen users: what a call costs before anything is computed
        {"name": "route_step", "op": "route", "tokens": 24, "experts": 64, "k": 4, "type": "bf16", "renorm": True, "plan": False, "masked": 0,
         "train": False},
        # a training batch over 256 ranks, with the arrays of the all-to-all and the gradient; a few experts are masked
        {"name": "route_batch_train", "op": "route", "tokens": 65536, "experts": 256, "k": 8, "type": "f32", "renorm": False, "plan": True,
         "masked": 3, "train": True},
        # rows packed as records of 8-bit values and their scales, in the order of the send buffer
        {"name": "quantise_dispatch", "op": "quantise", "form": "dispatch", "tokens": 16384, "hidden": 4096, "k": 4, "type": "bf16", "scale": "e8",
         "dropped": 100},
        # the experts' gated activation on the way to the second product, and its gradient; an odd number of rows
        {"name": "quantise_gated_train", "op": "quantise", "form": "gated", "tokens": 20011, "hidden": 1792, "k": 1, "type": "bf16", "scale": "f32",
         "dropped": 0},
        # one dense product of a generation step: the weights are read once and little else
        {"name": "matmul_step", "op": "matmul", "tokens": 40, "hidden": 2048, "out": 4096, "experts": 1, "skew": 0.0, "scale": "f32", "type": "bf16",
         "train": False},
        # the experts' first product on the ragged rows that an all-to-all brought
        {"name": "matmul_experts", "op": "matmul", "tokens": 16384, "hidden": 4096, "out": 3584, "experts": 64, "skew": 0.5, "scale": "e8",
         "type": "bf16", "train": False},
        # a training step's three products with the quantisation of what they read; odd rows, columns that are no multiple of 128
        {"name": "matmul_experts_train", "op": "matmul", "tokens": 12005, "hidden": 2048, "out": 2736, "experts": 8, "skew": 0.3, "scale": "f32",
         "type": "bf16", "train": True},
        # a prompt's dense product: bound by the matrix cores
        {"name": "matmul_prompt", "op": "matmul", "tokens": 16384, "hidden": 8192, "out": 8192, "experts": 1, "skew": 0.0, "scale": "e8",
         "type": "bf16", "train": False},
        # the sum over a token's experts in a generation step
        {"name": "combine_step", "op": "combine", "tokens": 24, "hidden": 2048, "k": 4, "type": "bf16", "dropped": 0, "train": False},
        # the same for a training batch with its gradient
        {"name": "combine_batch_train", "op": "combine", "tokens": 16384, "hidden": 4096, "k": 8, "type": "bf16", "dropped": 1000, "train": True},
        # the whole layer for one token
        {"name": "few_one_token", "op": "few", "tokens": 1, "hidden": 2048, "inner": 1024, "experts": 64, "k": 4, "weights": "f8", "scale": "f32"},
        # the whole layer for a few dozen users: nearly every expert's weights are read
        {"name": "few_forty_tokens", "op": "few", "tokens": 40, "hidden": 4096, "inner": 1536, "experts": 128, "k": 8, "weights": "f8", "scale": "e8"},
    ]


def _log(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["route", "quantise", "matmul", "matmul", "combine", "few"])
    if op == "route":
        experts = rng.choice([8, 16, 60, 64, 128, 200, 256])
        k = rng.choice([v for v in (1, 2, 4, 6, 8) if v <= experts])
        tokens = _log(rng, 1, 65000)
        return {"op": op, "tokens": tokens, "experts": experts, "k": k, "type": rng.choice(["bf16", "f32"]), "renorm": rng.random() < 0.5,
                "plan": tokens > 256 and rng.random() < 0.5, "masked": rng.choice([0, 0, 3]), "train": rng.random() < 0.5}
    if op == "quantise":
        if rng.random() < 0.5:
            return {"op": op, "form": "dispatch", "tokens": _log(rng, 16, 16000), "hidden": 64 * rng.randint(8, 64), "k": rng.choice([1, 2, 4]),
                    "type": rng.choice(["bf16", "f32"]), "scale": rng.choice(["f32", "e8"]), "dropped": rng.choice([0, 5])}
        return {"op": op, "form": "gated", "tokens": _log(rng, 16, 20000), "hidden": 16 * rng.randint(16, 112), "k": 1, "type": "bf16",
                "scale": rng.choice(["f32", "e8"]), "dropped": 0}
    if op == "matmul":
        train = rng.random() < 0.35
        experts = rng.choice([1, 1, 4, 8, 32])
        top = 10000 if train else 16000
        return {"op": op, "tokens": _log(rng, 64 if train else 1, top), "hidden": 16 * rng.randint(32, 256), "out": 16 * rng.randint(32, 256),
                "experts": experts, "skew": round(rng.uniform(0.0, 0.6), 2) if experts > 1 else 0.0, "scale": rng.choice(["f32", "e8"]),
                "type": rng.choice(["bf16", "bf16", "f32"]), "train": train}
    if op == "combine":
        return {"op": op, "tokens": _log(rng, 1, 16000), "hidden": 8 * rng.randint(64, 512), "k": rng.choice([1, 2, 4, 8]),
                "type": rng.choice(["bf16", "f32"]), "dropped": rng.choice([0, 1]), "train": rng.random() < 0.5}
    experts = rng.choice([8, 16, 60, 128])
    return {"op": "few", "tokens": _log(rng, 1, 64), "hidden": 128 * rng.randint(8, 32), "inner": 16 * rng.randint(32, 96), "experts": experts,
            "k": rng.choice([v for v in (1, 2, 4, 8) if v <= experts]), "weights": rng.choice(["f8", "f8", "bf16"]), "scale": rng.choice(["f32", "e8"])}


# ---------------------------------------------------------------------------------------------------- helpers of the plain forms


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _scales(peak, kind):
    """The scale of a block whose largest magnitude is `peak`, as a 32-bit value: peak / 448, or the smallest power of two that is not less."""
    s = (peak / torch.full_like(peak, 448.0)).clamp_min(2.0 ** -126)     # a division: a number would become a product with 1 / 448
    if kind == "e8":
        bits = s.view(torch.int32)
        s = (((bits + 0x7FFFFF) >> 23) << 23).view(torch.float32)
    return torch.where(peak == 0, torch.ones_like(s), s)


def _quantise(x, kind):
    """The last axis in blocks of 128: (e4m3 values, scales in 32 bits)."""
    n = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, _blocks(n) * BLOCK - n)).unflatten(-1, (-1, BLOCK))
    s = _scales(torch.where(x.isfinite(), x.abs(), 0.0).amax(-1), kind)
    return (x / s[..., None]).to(FLOAT8).flatten(-2)[..., :n], s


def _stored(s, kind):
    """Scales as they are kept: 32-bit values, or the exponent byte of a power of two."""
    return (s.view(torch.int32) >> 23).to(torch.uint8) if kind == "e8" else s


def _value(s, kind):
    return (s.to(torch.int32) << 23).view(torch.float32) if kind == "e8" else s


def _wide(q, s, kind, rows=1):
    """8-bit values times their scales, in 32 bits; `rows` rows share a scale."""
    s = _value(s, kind).repeat_interleave(BLOCK, -1)[..., :q.shape[-1]]
    if rows > 1:
        s = s.repeat_interleave(rows, -2)[..., :q.shape[-2], :]
    return q.float() * s


def _padded(rows, groups, most):
    """For ragged groups of rows: the row in every place of [groups, most], and whether there is one."""
    place = torch.arange(most, device=rows.device)
    return rows[:groups, None].long() + place, place < (rows[1:] - rows[:-1])[:, None]


# ---------------------------------------------------------------------------------------------------- inputs


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEVICE, dtype=dtype)


def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device=DEVICE)


def _some_slots(g, pairs, dropped):
    """The places of the pairs in a random order; the last `dropped` of them are not routed at all."""
    slots = torch.randperm(pairs, generator=g, device=DEVICE).to(torch.int32)
    return torch.where(slots < pairs - dropped, slots, -1)


def prepare_route(c, g):
    """type: of the logits; renorm: weights sum to one; plan: the all-to-all's arrays, for records of 1024 bytes;
    masked: that many experts of every seventh token have a logit of -inf, and all of every thousandth."""
    t, e, k = c["tokens"], c["experts"], c["k"]
    logits = _randn(g, t, e) * 2
    if c["masked"]:
        logits[::7, :c["masked"]] = -math.inf
        logits[5::1000] = -math.inf
    s = {"logits": logits.to(TYPES[c["type"]]), "dweights": _randn(g, t, k), "row_bytes": 1024, "workspace": None}
    s.update(experts=_empty(t, k, dtype=torch.int32), weights=_empty(t, k), slots=_empty(t, k, dtype=torch.int32),
             rows=_empty(e + 1, dtype=torch.int32), dlogits=torch.empty_like(s["logits"]), plan=(None,) * 4)
    if c["plan"]:
        s["plan"] = tuple(_empty(e, e, dtype=d) for d in (torch.int32, torch.int64) * 2)
    return s


def prepare_quantise(c, g):
    """form: dispatch (every row to the slots of its k pairs, as records of values and scales) or gated (silu(gate) * up, with the
    gradient); dropped: pairs without a slot."""
    t, h, k = c["tokens"], c["hidden"], c["k"]
    nb = _blocks(h)
    if c["form"] == "dispatch":
        out = t * k - c["dropped"]
        record = -(-(h + nb * (1 if c["scale"] == "e8" else 4)) // 16) * 16
        x = _randn(g, t, h) * torch.exp(_randn(g, t, 1))
        return {"x": x.to(TYPES[c["type"]]), "slots": _some_slots(g, t * k, c["dropped"]), "records": torch.zeros(out, record, dtype=torch.uint8, device=DEVICE)}
    return {"x": _randn(g, t, 2 * h, dtype=torch.bfloat16) * 2, "dh": _randn(g, t, h, dtype=torch.bfloat16),
            "q": _empty(t, h, dtype=torch.uint8), "s": _empty(t, nb, dtype=torch.uint8 if c["scale"] == "e8" else torch.float32),
            "dx": _empty(t, 2 * h, dtype=torch.bfloat16)}


def _weights8(g, kind, *shape):
    """8-bit weights as a program keeps them, with a scale for 128 x 128 of them."""
    q = (_randn(g, *shape, dtype=torch.bfloat16) * 64).to(FLOAT8)
    s = torch.exp2(torch.randint(-14, -10, (*shape[:-2], _blocks(shape[-2]), _blocks(shape[-1])), generator=g, device=DEVICE).float())
    if kind == "f32":
        s *= 1 + torch.rand(s.shape, generator=g, device=DEVICE)
    return q, _stored(s, kind)


def prepare_matmul(c, g):
    """tokens rows of `hidden` in ragged groups of the experts, times each expert's [out, hidden] weights; type: of the product;
    skew: how unevenly the rows are spread; train: inputs in bf16, and the three products with their quantisation."""
    m, n, kk, e = c["tokens"], c["out"], c["hidden"], c["experts"]
    share = torch.arange(1, e + 1, device=DEVICE).float() ** -c["skew"]
    which = torch.multinomial(share, m, replacement=True, generator=g)
    rows = torch.zeros(e + 1, dtype=torch.int32, device=DEVICE)
    rows[1:] = torch.cumsum(torch.bincount(which, minlength=e), 0)
    w, ws = _weights8(g, c["scale"], e, n, kk)
    s = {"rows": rows, "most": int((rows[1:] - rows[:-1]).max()), "w": w, "ws": ws, "y": _empty(m, n, dtype=TYPES[c["type"]])}
    x = _randn(g, m, kk, dtype=torch.bfloat16)
    if not c["train"]:
        q, sc = _quantise(x, c["scale"])
        return dict(s, x=q.contiguous(), xs=_stored(sc, c["scale"]))      # rows of `hidden` values back to back, as `run` says
    st = torch.uint8 if c["scale"] == "e8" else torch.float32
    wide = _blocks(m) * BLOCK + e * BLOCK                        # room for every group's rows, in whole blocks of 128
    s.update(x=x, dy=_randn(g, m, n, dtype=torch.bfloat16), wt=w.transpose(1, 2).contiguous(), wts=ws.transpose(1, 2).contiguous(),
             dx=_empty(m, kk, dtype=TYPES[c["type"]]), dw=_empty(e, n, kk))
    for name, cols in (("x", kk), ("dy", n)):
        s.update({name + "_q": _empty(m, cols, dtype=torch.uint8), name + "_s": _empty(m, _blocks(cols), dtype=st),
                  name + "_tq": _empty(cols, wide, dtype=torch.uint8), name + "_ts": _empty(cols, wide // BLOCK, dtype=st)})
    return s


def prepare_combine(c, g):
    """dropped: pairs that were not routed."""
    t, h, k = c["tokens"], c["hidden"], c["k"]
    ty, rows = TYPES[c["type"]], t * k - c["dropped"]
    return {"y": _randn(g, rows, h).to(ty), "slots": _some_slots(g, t * k, c["dropped"]).view(t, k), "weights": torch.rand(t, k, generator=g, device=DEVICE),
            "dout": _randn(g, t, h).to(ty), "out": _empty(t, h, dtype=ty), "dy": _empty(rows, h, dtype=ty), "dweights": _empty(t, k)}


def prepare_few(c, g):
    """weights: f8 with a scale for 128 x 128, or bf16; gate rows come before up rows; inner: columns between the two products."""
    t, h, f, e = c["tokens"], c["hidden"], c["inner"], c["experts"]
    s = {"x": _randn(g, t, h, dtype=torch.bfloat16), "logits": _randn(g, t, e) * 2, "out": _empty(t, h, dtype=torch.bfloat16), "workspace": None,
         "s1": None, "s2": None}
    for name, shape in (("1", (e, 2 * f, h)), ("2", (e, h, f))):
        if c["weights"] == "f8":
            s["w" + name], s["s" + name] = _weights8(g, c["scale"], *shape)
        else:
            s["w" + name] = _randn(g, *shape, dtype=torch.bfloat16) * 0.02
    return s


def prepare(case, seed):
    s = globals()["prepare_" + case["op"]](case, _gen(seed))
    s["case"] = case
    return s


# ---------------------------------------------------------------------------------------------------- plain forms


def _choose(logits, k, renorm):
    """(softmax, experts, weights): the k largest eligible logits, ties to the lowest index."""
    l = logits.float()
    l = torch.where(l.isnan(), -math.inf, l)
    top = l.amax(-1, keepdim=True)
    p = torch.exp(l - torch.where(top == -math.inf, 0.0, top))
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-30)
    order = torch.sort(l, dim=-1, descending=True, stable=True)
    there = order.values[:, :k] > -math.inf
    experts = torch.where(there, order.indices[:, :k], -1)
    w = torch.where(there, p.gather(1, order.indices[:, :k]), 0.0)
    if renorm:
        w = w / w.sum(-1, keepdim=True).clamp_min(1e-30)
    return p, experts.to(torch.int32), w


def plain_route(s, c):
    t, e, k = c["tokens"], c["experts"], c["k"]
    p, experts, w = _choose(s["logits"], k, c["renorm"])
    pairs = experts.reshape(-1).long()
    shard = -(-t // e) if c["plan"] else t
    rank = torch.arange(t, device=DEVICE).repeat_interleave(k) // shard
    order = torch.sort(torch.where(pairs < 0, e * e, rank * e + pairs), stable=True).indices
    slots = torch.empty_like(pairs)
    slots[order] = torch.arange(t * k, device=DEVICE)
    counts = torch.bincount(torch.where(pairs < 0, e, pairs), minlength=e + 1)[:e]
    out = {"experts": experts, "weights": w, "slots": torch.where(pairs < 0, -1, slots).to(torch.int32).view(t, k),
           "rows": torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0)).to(torch.int32)}
    if c["plan"]:
        cnt = torch.bincount(torch.where(pairs < 0, e * e, rank * e + pairs), minlength=e * e + 1)[:e * e].view(e, e) * s["row_bytes"]
        back = cnt.t().contiguous()
        out["plan"] = [v for m in (cnt, back) for v in (m.to(torch.int32), (torch.cumsum(m.view(-1), 0) - m.view(-1)).view(e, e))]
    if c["train"]:
        g = torch.zeros_like(p).scatter_add_(1, experts.clamp_min(0).long(), torch.where(experts < 0, 0.0, s["dweights"]))
        if c["renorm"]:
            p = torch.zeros_like(p).scatter_add_(1, experts.clamp_min(0).long(), w)
        out["dlogits"] = (p * (g - (g * p).sum(-1, keepdim=True))).to(s["logits"].dtype)
    return out


def plain_quantise(s, c):
    if c["form"] == "dispatch":
        q, sc = _quantise(s["x"], c["scale"])
        sc, slots = _stored(sc, c["scale"]), s["slots"].long()
        token = torch.arange(c["tokens"], device=DEVICE).repeat_interleave(c["k"])
        rows = s["records"].shape[0]
        token = torch.zeros(rows + 1, dtype=torch.int64, device=DEVICE).scatter_(0, torch.where(slots < 0, rows, slots), token)[:rows]
        return {"q": q.view(torch.uint8)[token].view(FLOAT8), "s": sc[token]}
    h = c["hidden"]
    gate, up = s["x"][:, :h].float(), s["x"][:, h:].float()
    sig = 1 / (1 + torch.exp(-gate))
    q, sc = _quantise(gate * sig * up, c["scale"])
    dh = s["dh"].float()
    return {"q": q, "s": _stored(sc, c["scale"]).to(torch.float32 if c["scale"] == "f32" else torch.uint8),
            "dx": torch.cat([dh * up * sig * (1 + gate * (1 - sig)), dh * gate * sig], 1).to(torch.bfloat16)}


def _spread(s, c, x):
    """Rows of ragged groups in [experts, most] places, zero where there is none."""
    at, there = _padded(s["rows"], c["experts"], s["most"])
    return torch.where(there[..., None], x[at.clamp_max(x.shape[0] - 1)], 0), there


def _product(s, c, x, w):
    x, there = _spread(s, c, x)
    return torch.bmm(x, w.transpose(1, 2).contiguous())[there]


def plain_matmul(s, c):
    w = _wide(s["w"], s["ws"], c["scale"], BLOCK)
    if not c["train"]:
        return _product(s, c, _wide(s["x"], s["xs"], c["scale"]), w).to(s["y"].dtype)
    again = lambda v: _wide(*_quantise(v, "f32"), "f32") if c["scale"] == "f32" else _wide(*_quantise(v, "e8"), "f32")  # noqa: E731
    y, dx = _product(s, c, again(s["x"]), w), _product(s, c, again(s["dy"]), w.transpose(1, 2))
    by_rows = [again(_spread(s, c, v)[0].transpose(1, 2).contiguous()) for v in (s["dy"], s["x"])]
    return {"y": y.to(s["y"].dtype), "dx": dx.to(s["y"].dtype), "dw": torch.bmm(by_rows[0], by_rows[1].transpose(1, 2).contiguous())}


def plain_combine(s, c):
    slots, w = s["slots"].long(), s["weights"]
    there = (slots >= 0)[..., None]
    y = torch.where(there, s["y"][slots.clamp_min(0)].float(), 0.0)
    out = {"out": (w[..., None] * y).sum(1).to(s["out"].dtype)}
    if c["train"]:
        dout = s["dout"].float()
        rows = s["y"].shape[0]
        dy = torch.empty(rows + 1, c["hidden"], dtype=s["out"].dtype, device=DEVICE)
        dy[torch.where(slots < 0, rows, slots).view(-1)] = (w[..., None] * dout[:, None]).to(dy.dtype).flatten(0, 1)
        out.update(dy=dy[:rows], dweights=(dout[:, None] * y).sum(-1))
    return out


def plain_few(s, c):
    t, f, e = c["tokens"], c["inner"], c["experts"]
    _, experts, w = _choose(s["logits"], c["k"], True)
    x = s["x"].float()
    if t * c["k"] <= e:                                          # the chosen experts' weights, once for every pair
        at = experts.clamp_min(0).view(-1).long()
        x = x.repeat_interleave(c["k"], 0)[:, None]
    else:                                                        # all experts on all tokens
        at = torch.arange(e, device=DEVICE)
        x = x.expand(e, *x.shape)
    part = lambda n: s["w" + n][at].float() if s["s" + n] is None else _wide(  # noqa: E731
        s["w" + n].view(torch.uint8)[at].view(FLOAT8), s["s" + n][at], c["scale"], BLOCK)
    a = torch.bmm(x, part("1").transpose(1, 2).contiguous())
    gate, up = a[..., :f], a[..., f:]
    y = torch.bmm(gate / (1 + torch.exp(-gate)) * up, part("2").transpose(1, 2).contiguous())
    if t * c["k"] <= e:
        y = y.view(t, c["k"], -1)
    else:
        y = y[experts.clamp_min(0).long(), torch.arange(t, device=DEVICE)[:, None]]
    return (torch.where(experts < 0, 0.0, w)[..., None] * y).sum(1).to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------------- the framework's


def _tuna():
    import paper_2411_02581_amd as tuna
    return tuna


def _ok(tuna, *codes):
    for rc in codes:
        if rc != tuna.TUNA_OK:
            raise RuntimeError(tuna.tuna_strerror(rc))


def own_route(s, c):
    tuna = _tuna()
    t, e, k = c["tokens"], c["experts"], c["k"]
    ty, flags = tuna.TUNA_BF16 if c["type"] == "bf16" else tuna.TUNA_F32, tuna.TUNA_ROUTE_RENORM if c["renorm"] else 0
    if s["workspace"] is None:
        rc, size = tuna.tuna_moe_route_workspace(t, e, k, c["plan"])
        _ok(tuna, rc)
        s["workspace"] = _empty(max(size, 16), dtype=torch.uint8)
    _ok(tuna, tuna.tuna_moe_route(s["logits"], ty, e, t, e, k, flags, s["experts"], s["weights"], s["slots"], s["rows"], s["row_bytes"], *s["plan"],
                                  s["workspace"], s["workspace"].numel()))
    out = {"experts": s["experts"], "weights": s["weights"], "slots": s["slots"], "rows": s["rows"]}
    if c["plan"]:
        out["plan"] = list(s["plan"])
    if c["train"]:
        _ok(tuna, tuna.tuna_moe_route_grad(s["logits"], ty, e, t, e, k, flags, s["experts"], s["weights"], s["dweights"], s["dlogits"], e))
        out["dlogits"] = s["dlogits"]
    return out


def _kind(tuna, c):
    return tuna.TUNA_SCALE_E8 if c["scale"] == "e8" else tuna.TUNA_SCALE_F32


def own_quantise(s, c):
    tuna = _tuna()
    t, h, nb = c["tokens"], c["hidden"], _blocks(c["hidden"])
    if c["form"] == "dispatch":
        rec = s["records"]
        rows, size = rec.shape
        scales = rec[:, h:h + nb] if c["scale"] == "e8" else rec[:, h:h + 4 * nb].view(torch.float32)
        ty = tuna.TUNA_BF16 if c["type"] == "bf16" else tuna.TUNA_F32
        _ok(tuna, tuna.tuna_fp8_quantize(s["x"], ty, h, t, h, tuna.TUNA_ACT_NONE, s["slots"], c["k"], rows, rec, size, scales, scales.stride(0), _kind(tuna, c)))
        return {"q": rec[:, :h].view(FLOAT8), "s": scales}
    _ok(tuna, tuna.tuna_fp8_quantize(s["x"], tuna.TUNA_BF16, 2 * h, t, h, tuna.TUNA_ACT_SWIGLU, None, 1, t, s["q"], h, s["s"], nb, _kind(tuna, c)),
        tuna.tuna_moe_swiglu_grad(s["x"], tuna.TUNA_BF16, 2 * h, s["dh"], h, t, h, s["dx"], 2 * h))
    return {"q": s["q"].view(FLOAT8), "s": s["s"], "dx": s["dx"]}


def own_matmul(s, c):
    tuna = _tuna()
    m, n, kk, e = c["tokens"], c["out"], c["hidden"], c["experts"]
    ty, kind, nk, nn = tuna.TUNA_BF16 if c["type"] == "bf16" else tuna.TUNA_F32, _kind(tuna, c), _blocks(kk), _blocks(n)
    rows = s["rows"] if e > 1 else None
    x, xs = (s["x_q"], s["x_s"]) if c["train"] else (s["x"], s["xs"])
    if c["train"]:
        wide = s["x_tq"].shape[1]
        for name, cols in (("x", kk), ("dy", n)):
            _ok(tuna, tuna.tuna_fp8_quantize(s[name], tuna.TUNA_BF16, cols, m, cols, tuna.TUNA_ACT_NONE, None, 1, m, s[name + "_q"], cols, s[name + "_s"],
                                             _blocks(cols), kind),
                tuna.tuna_fp8_quantize_columns(s[name], tuna.TUNA_BF16, cols, m, cols, rows, e, s[name + "_tq"], wide, s[name + "_ts"], wide // BLOCK, kind))
    _ok(tuna, tuna.tuna_fp8_matmul(x, kk, xs, nk, s["w"], kk, n * kk, s["ws"], nk, nn * nk, kind, rows, e, s["y"], ty, n, m, n, kk))
    if not c["train"]:
        return s["y"]
    _ok(tuna, tuna.tuna_fp8_matmul(s["dy_q"], n, s["dy_s"], nn, s["wt"], n, n * kk, s["wts"], nn, nn * nk, kind, rows, e, s["dx"], ty, kk, m, kk, n),
        tuna.tuna_fp8_matmul_grad_w(s["dy_tq"], wide, s["dy_ts"], wide // BLOCK, s["x_tq"], wide, s["x_ts"], wide // BLOCK, kind, rows, e,
                                    s["dw"], tuna.TUNA_F32, kk, n * kk, m, n, kk))
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


def own_combine(s, c):
    tuna = _tuna()
    t, h, k, rows = c["tokens"], c["hidden"], c["k"], s["y"].shape[0]
    ty = tuna.TUNA_BF16 if c["type"] == "bf16" else tuna.TUNA_F32
    _ok(tuna, tuna.tuna_moe_combine(s["y"], ty, h, rows, s["slots"], s["weights"], t, k, h, s["out"], ty, h))
    if not c["train"]:
        return {"out": s["out"]}
    _ok(tuna, tuna.tuna_moe_combine_grad(s["dout"], ty, h, s["y"], ty, h, rows, s["slots"], s["weights"], t, k, h, s["dy"], h, s["dweights"]))
    return {"out": s["out"], "dy": s["dy"], "dweights": s["dweights"]}


def own_few(s, c):
    tuna = _tuna()
    t, h, f, e, k = c["tokens"], c["hidden"], c["inner"], c["experts"], c["k"]
    if s["workspace"] is None:
        rc, size = tuna.tuna_moe_few_workspace(t, h, f, e, k)
        _ok(tuna, rc)
        s["workspace"] = _empty(size, dtype=torch.uint8)
    wt = tuna.TUNA_F8 if c["weights"] == "f8" else tuna.TUNA_BF16
    _ok(tuna, tuna.tuna_moe_few(s["x"], h, t, h, s["logits"], tuna.TUNA_F32, e, e, k, tuna.TUNA_ROUTE_RENORM, s["w1"], s["s1"], s["w2"], s["s2"], f, wt,
                                _kind(tuna, c), s["out"], tuna.TUNA_BF16, h, s["workspace"], s["workspace"].numel()))
    return s["out"]


def run(state):
    c = state["case"]
    return globals()[("own_" if own else "plain_") + c["op"]](state, c)


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits


def _exact_softmax(logits):
    l = logits.double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    return torch.softmax(l, -1).nan_to_num(nan=0.0)


def _exact_top(p, l, k):
    """Where an expert is among the k first of its token: fewer than k come before it."""
    ahead = torch.empty_like(p, dtype=torch.int64)
    for at in range(0, p.shape[0], 1024):
        v = l[at:at + 1024].double()
        first = torch.arange(v.shape[1], device=v.device)
        ahead[at:at + 1024] = ((v[:, None] > v[:, :, None]) | ((v[:, None] == v[:, :, None]) & (first < first[:, None]))).sum(-1)
    return (ahead < k) & (l > -math.inf), ahead


def _exact_weights(c, logits):
    p = _exact_softmax(logits)
    chosen, ahead = _exact_top(p, logits.float(), c["k"])
    w = torch.where(chosen, p, 0.0)
    if c.get("renorm", True):
        w = (w / w.sum(-1, keepdim=True)).nan_to_num(nan=0.0)
    return p, chosen, ahead, w


def exact_route(s, c):
    p, chosen, ahead, w = _exact_weights(c, s["logits"])
    at = torch.where(chosen, ahead, c["k"])
    to = lambda v: torch.zeros(v.shape[0], c["k"] + 1, dtype=v.dtype, device=v.device).scatter_(1, at, v)[:, :c["k"]]  # noqa: E731
    out = {"experts": None, "weights": to(w), "slots": None, "rows": None}
    if c["plan"]:
        out["plan"] = [None] * 4
    if c["train"]:
        g = torch.where(chosen, s["dweights"].double().gather(1, at.clamp_max(c["k"] - 1)), 0.0)
        p = w if c["renorm"] else p
        out["dlogits"] = p * g - p * (p * g).sum(-1, keepdim=True)
    return out


def _exact_blocks(x, kind):
    """Values as 8 bits and a 32-bit scale hold them, in 64 bits."""
    n = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    s = (top / 448).float().double()
    if kind == "e8":
        m, e = torch.frexp(s)
        s = torch.ldexp(torch.ones_like(s), torch.where(m == 0.5, e - 1, e))
    s = torch.where(top == 0, 1.0, s)
    return ((x / s).to(torch.float32).to(FLOAT8).double()).flatten(-2)[..., :n], s.squeeze(-1)


def exact_quantise(s, c):
    if c["form"] == "dispatch":
        q, sc = _exact_blocks(s["x"], c["scale"])
        slots = s["slots"].long()
        rows = s["records"].shape[0]
        source = torch.empty(rows, dtype=torch.int64, device=DEVICE)
        source[slots[slots >= 0]] = (slots >= 0).nonzero().squeeze(1) // c["k"]
        return {"q": q[source], "s": None if c["scale"] == "e8" else sc[source]}
    a, b = s["x"].double().chunk(2, 1)
    act = torch.sigmoid(a) * a
    d = s["dh"].double()
    slope = torch.sigmoid(a) + act * torch.sigmoid(-a)
    q, sc = _exact_blocks(act * b, c["scale"])
    return {"q": q, "s": None if c["scale"] == "e8" else sc, "dx": torch.cat([d * b * slope, d * act], 1)}


def _exact_wide(q, s, kind, rows):
    s = torch.exp2(s.double() - 127) if kind == "e8" else s.double()
    i = torch.arange(q.shape[-2], device=q.device) // rows
    j = torch.arange(q.shape[-1], device=q.device) // BLOCK
    return q.double() * s[..., i, :][..., j]


def exact_matmul(s, c):
    kind, rows, e = c["scale"], s["rows"].tolist(), c["experts"]
    both = lambda v: (lambda q, sc: q * sc.repeat_interleave(BLOCK, -1)[..., :v.shape[-1]])(*_exact_blocks(v, kind))  # noqa: E731
    x = both(s["x"]) if c["train"] else _exact_wide(s["x"], s["xs"], kind, 1)
    d = both(s["dy"]) if c["train"] else None
    y, dx, dw = [], [], []
    for i in range(e):
        a, b = rows[i], rows[i + 1]
        w = _exact_wide(s["w"][i], s["ws"][i], kind, BLOCK)
        y.append(x[a:b] @ w.t())
        if c["train"]:
            dx.append(d[a:b] @ w)
            dw.append(both(s["dy"][a:b].t()) @ both(s["x"][a:b].t()).t())
    return {"y": torch.cat(y), "dx": torch.cat(dx), "dw": torch.stack(dw)} if c["train"] else torch.cat(y)


def exact_combine(s, c):
    t, k = s["slots"].shape
    y = torch.cat([s["y"].double(), torch.zeros(1, c["hidden"], dtype=torch.float64, device=DEVICE)])
    out = torch.zeros(t, c["hidden"], dtype=torch.float64, device=DEVICE)
    d, dy, dw = s["dout"].double(), torch.zeros_like(y), []
    for j in range(k):
        at, w = s["slots"][:, j].long(), s["weights"][:, j:j + 1].double()
        out += w * y[at]                                         # slot -1 is the row of zeros at the end
        dy[at] = w * d
        dw.append((d * y[at]).sum(-1))
    return {"out": out, "dy": dy[:-1], "dweights": torch.stack(dw, 1)} if c["train"] else {"out": out}


def exact_few(s, c):
    f = c["inner"]
    _, chosen, _, w = _exact_weights(c, s["logits"])
    x, out = s["x"].double(), torch.zeros(c["tokens"], c["hidden"], dtype=torch.float64, device=DEVICE)
    for e in chosen.any(0).nonzero().squeeze(1).tolist():
        w1, w2 = ((s["w" + n][e].double() if s["s" + n] is None else _exact_wide(s["w" + n][e], s["s" + n][e], c["scale"], BLOCK)) for n in "12")
        a = x @ w1.t()
        out += w[:, e:e + 1] * ((a[:, :f] * torch.sigmoid(a[:, :f]) * a[:, f:]) @ w2.t())
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return globals()["exact_" + case["op"]](s, case)


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without


def _width(c):
    return 2 if c.get("type") == "bf16" else 4


def work(case):
    c = case
    t, k, h, e = c["tokens"], c.get("k", 1), c.get("hidden", 0), c.get("experts", 1)
    nb, one = _blocks(h), 1 if c.get("scale") == "e8" else 4
    if c["op"] == "route":
        size = t * e * _width(c) + 12 * t * k + 4 * (e + 1) + (24 * e * e if c["plan"] else 0)
        if c["train"]:                                           # the logits are read once more or kept: once is enough
            size += 4 * t * k + t * e * _width(c)
        return {"bytes": float(size), "flops": 4.0 * t * e}
    if c["op"] == "quantise":
        if c["form"] == "dispatch":
            return {"bytes": float(t * h * _width(c) + 4 * t * k + (t * k - c["dropped"]) * (h + one * nb)), "flops": 2.0 * t * h}
        return {"bytes": float(t * h * 4 + t * (h + one * nb) + t * h * 2 + t * h * 4), "flops": 20.0 * t * h}
    if c["op"] == "matmul":
        n = c["out"]
        w = min(e, t) * (n * h + one * nb * _blocks(n))
        if not c["train"]:
            return {"bytes": float(t * (h + one * nb) + w + t * n * _width(c)), "flops": 2.0 * t * n * h}
        return {"bytes": float(2 * t * (h + n) + 2 * w + t * (h + n) * _width(c) + 4 * e * n * h), "flops": 6.0 * t * n * h}
    if c["op"] == "combine":
        rows = t * k - c["dropped"]
        size = rows * h * _width(c) + 8 * t * k + t * h * _width(c)
        if c["train"]:
            size += t * h * _width(c) + rows * h * _width(c) + 4 * t * k
        return {"bytes": float(size), "flops": (6.0 if c["train"] else 2.0) * rows * h}
    f, some = c["inner"], e * (1 - (1 - k / e) ** t)             # experts that are chosen, on average
    each = 3 * f * h * (2 if c["weights"] == "bf16" else 1)
    return {"bytes": float(some * each + 4 * t * h + 4 * t * e), "flops": 6.0 * t * k * f * h}
