"""Performance cases of the operators around a LookME layer: the residual sum
with the norm, rows grouped by expert, products grouped by expert, and
products of few rows with 4-bit weights.

``own`` chooses between the plain form (elementary torch operations in 32
bits) and the library's entry points.  Kinds:

  norm     H + weighted parts, RMS norm, outputs in the storage type and in
           e4m3 with a scale a row
  group    stable grouping of entries by a picked id
  grouped  y = x W_g^T for rows grouped by g, plain or gate and up (SwiGLU),
           bf16, float32 or e4m3 with scales
  quant    y = x W^T with 4-bit weights, scales (and zero points) by groups
"""

import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0
TINY = 2.0 ** -126       # the smallest scale a row can get
EPS = 1e-6
GIB = 1 << 30
MOST_FLOPS = 1.2e12      # of a drawn case: no more than the largest listed one
MOST_BYTES = 1.1 * GIB


def _norm(**kw):
    c = dict(kind="norm", dtype="bf16", n=1, d=2048, parts=1, weighted=False, out=True,
             quant=False)
    c.update(kw)
    return c


def _group(**kw):
    c = dict(kind="group", n=512, groups=128, zipf=0.0, dropped=0)
    c.update(kw)
    return c


def _grouped(**kw):
    c = dict(kind="grouped", dtype="bf16", tokens=16, picks=8, groups=128, d_in=2048, d_out=1024,
             zipf=0.0, swiglu=False, gather=True, scatter=False)
    c.update(kw)
    return c


def _quant(**kw):
    c = dict(kind="quant", dtype="bf16", n=1, d_in=2048, d_out=2048, group=128, zero=False,
             swiglu=False, add=False)
    c.update(kw)
    return c


def listed():
    return [
        # one decoded token: the add after attention and the norm before the next product
        _norm(name="norm_token"),
        # prefill of a batch of image crops: the norm feeds products in 8 bits
        _norm(name="norm_prefill_quant", n=23040, out=False, quant=True),
        # the weighted outputs of eight experts a token come back into the hidden states
        _norm(name="norm_combine_quant", n=8192, d=4096, parts=8, weighted=True, quant=True),
        # a decode step's picks, 64 sequences of eight experts each
        _group(name="group_decode"),
        # a whole batch's picks over a thousand scenes, a few of them masked out
        _group(name="group_scenes", n=262144, groups=1024, zipf=1.0, dropped=2),
        # a decode step: nearly every expert has a row or two, so the weights stream
        _grouped(name="grouped_decode", swiglu=True),
        # float32, ragged sizes, rows already in group order
        _grouped(name="grouped_f32_ragged", dtype="f32", tokens=3001, picks=1, groups=13,
                 d_in=1160, d_out=840, gather=False),
        # prefill: experts of uneven popularity, outputs back in the entries' order
        _grouped(name="grouped_prefill", tokens=8192, groups=64, d_out=2048, zipf=0.6,
                 scatter=True),
        # the largest: prefill in 8 bits
        _grouped(name="grouped_prefill_e4m3", dtype="e4m3", tokens=16384, picks=2, groups=16,
                 d_in=4096, d_out=4096),
        # one decoded token through a square projection
        _quant(name="quant_token"),
        # four sequences' tokens through gate and up
        _quant(name="quant_swiglu", n=4, d_in=4096, d_out=8192, zero=True, swiglu=True),
        # float32 states, short groups, the residual added
        _quant(name="quant_f32_rows", dtype="f32", n=16, d_in=4128, d_out=2056, group=32,
               zero=True, add=True),
    ]


def _log(rng, lo, hi, step=1):
    """A size between lo and hi, spread over the logarithm, a multiple of step."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "group", "grouped", "grouped", "grouped", "quant",
                           "quant"])
        if kind == "norm":
            quant = rng.random() < 0.6
            parts = rng.choice([0, 1, 1, 2, 4, 8])
            c = _norm(dtype=rng.choice(["bf16", "bf16", "f32"]), n=_log(rng, 1, 32768),
                      d=_log(rng, 64, 8192, 8), parts=parts,
                      weighted=parts > 0 and rng.random() < 0.5, quant=quant,
                      out=not quant or rng.random() < 0.5)
        elif kind == "group":
            c = _group(n=_log(rng, 1, 262144), groups=_log(rng, 1, 4096),
                       zipf=rng.choice([0.0, 0.6, 1.0]), dropped=rng.choice([0, 0, 2, 30]))
        elif kind == "grouped":
            groups = _log(rng, 1, 256)
            picks = rng.choice([1, 2, 4, 8])
            gather = rng.random() < 0.7
            c = _grouped(dtype=rng.choice(["bf16", "bf16", "e4m3", "f32"]),
                         tokens=_log(rng, 1, 16384), picks=min(picks, groups), groups=groups,
                         d_in=_log(rng, 128, 4096, 16), d_out=_log(rng, 64, 4096, 8),
                         zipf=rng.choice([0.0, 0.3, 0.6]), swiglu=rng.random() < 0.4,
                         gather=gather, scatter=gather and rng.random() < 0.5)
            if c["dtype"] == "f32" and work(c)["flops"] > 1e11:
                continue
        else:
            swiglu = rng.random() < 0.4
            group = rng.choice([32, 64, 128, 128])
            c = _quant(dtype=rng.choice(["bf16", "bf16", "f32"]), n=_log(rng, 1, 64),
                       d_in=_log(rng, 256, 8192, group), d_out=_log(rng, 64, 8192, 8),
                       group=group, zero=rng.random() < 0.5, swiglu=swiglu,
                       add=not swiglu and rng.random() < 0.5)
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 17)
    return g


def _randn(g, shape, std, dtype):
    """N(0, std^2), drawn in float32 slices of the first dimension."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    rows = max(1, (1 << 26) // max(1, math.prod(shape[1:])))
    for a in range(0, shape[0], rows):
        b = min(shape[0], a + rows)
        t = torch.randn((b - a, *shape[1:]), generator=g, device="cuda")
        out[a:b] = t.mul_(std).to(dtype)
    return out


def _popularity(g, groups, s):
    """log-probabilities of the groups: rank^-s in a random order"""
    ranks = torch.arange(1, groups + 1, device="cuda", dtype=torch.float32)
    return (-s * ranks.log())[torch.randperm(groups, generator=g, device="cuda")]


def _picks(g, tokens, picks, groups, s):
    """[tokens, picks] distinct groups of every token, by popularity"""
    logp = _popularity(g, groups, s)
    u = torch.rand((tokens, groups), generator=g, device="cuda").clamp_(1e-20, 1 - 1e-7)
    return torch.topk(logp - torch.log(-torch.log(u)), picks, dim=1).indices.to(torch.int32)


def _quantized_rows(w):
    """e4m3 rows of w with a float32 scale each"""
    scale = (w.float().abs().amax(-1) / E4M3_MAX).clamp_min(TINY)
    return (w.float() / scale[..., None]).to(DTYPE["e4m3"]), scale


def _inputs(c, seed):
    g = _gen(seed)
    kind, s = c["kind"], {}
    if kind == "norm":
        dt, n, d, parts = DTYPE[c["dtype"]], c["n"], c["d"], c["parts"]
        s["hidden"] = _randn(g, (n, d), 2.0, dt)
        s["weight"] = (1 + _randn(g, (d,), 0.2, torch.float32)).to(dt)
        if parts:
            s["add"] = _randn(g, (n, parts, d), 0.5, dt)
        if c["weighted"]:
            s["part_w"] = torch.softmax(_randn(g, (n, parts), 1.0, torch.float32), 1)
    elif kind == "group":
        logp = _popularity(g, c["groups"], c["zipf"])
        p = torch.multinomial(torch.softmax(logp, 0), c["n"], replacement=True, generator=g)
        lost = torch.rand((c["n"],), generator=g, device="cuda") < c["dropped"] / 100
        s["pick"] = torch.where(lost, -1, p).to(torch.int32)
    elif kind == "grouped":
        G, n, k = c["groups"], c["tokens"], c["picks"]
        pick = _picks(g, n, k, G, c["zipf"]).reshape(-1).long()
        s["rows"] = torch.argsort(pick, stable=True).to(torch.int32)
        s["offsets"] = torch.cat([pick.new_zeros(1), torch.bincount(pick, minlength=G).cumsum(0)]
                                 ).to(torch.int32)
        quant = c["dtype"] == "e4m3"
        dt = torch.bfloat16 if quant else DTYPE[c["dtype"]]
        s["x"] = _randn(g, (n if c["gather"] else n * k, c["d_in"]), 1.0, dt)
        for name in ("w", "w_up")[:2 if c["swiglu"] else 1]:
            w = _randn(g, (G, c["d_out"], c["d_in"]), c["d_in"] ** -0.5, dt)
            s[name] = w
            if quant:
                q = torch.empty(w.shape, dtype=DTYPE["e4m3"], device="cuda")
                scale = torch.empty(w.shape[:2], device="cuda")
                for i in range(G):
                    q[i], scale[i] = _quantized_rows(w[i])
                s[name], s[name + "_scale"] = q, scale
        if quant:
            s["x"], s["x_scale"] = _quantized_rows(s["x"])
    else:
        dt, N, K, groups = DTYPE[c["dtype"]], c["d_out"], c["d_in"], c["d_in"] // c["group"]
        s["x"] = _randn(g, (c["n"], K), 1.0, dt)
        for name in ("w", "up")[:2 if c["swiglu"] else 1]:
            s[name] = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda",
                                    dtype=torch.uint8)
            u = torch.rand((N, groups), generator=g, device="cuda")
            s[name + "_scale"] = ((0.5 + u) * 0.2 * K ** -0.5).to(dt)
            if c["zero"]:
                s[name + "_zero"] = torch.randint(5, 12, (N, groups), generator=g, device="cuda",
                                                  dtype=torch.uint8)
        if c["add"]:
            s["add"] = _randn(g, (c["n"], N), 1.0, dt)
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    kind = c["kind"]
    empty = lambda shape, dt: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    # the buffers that a program keeps for its outputs
    if kind == "norm":
        n, d, dt = c["n"], c["d"], DTYPE[c["dtype"]]
        s["hidden_out"] = empty((n, d), dt)
        s["out"] = empty((n, d), dt) if c["out"] else None
        s["out_quant"] = empty((n, d), DTYPE["e4m3"]) if c["quant"] else None
        s["scale_out"] = empty((n,), torch.float32) if c["quant"] else None
    elif kind == "group":
        s["rows_out"] = torch.full((c["n"],), -1, dtype=torch.int32, device="cuda")
        s["offsets_out"] = empty((c["groups"] + 1,), torch.int32)
    elif kind == "grouped":
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        s["out"] = empty((c["tokens"] * c["picks"], c["d_out"]), dt)
    else:
        s["out"] = empty((c["n"], c["d_out"]), DTYPE[c["dtype"]])
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _plain_norm(c, s):
    h = s["hidden"].float()
    if c["parts"]:
        a = s["add"].float()
        h = h + (a * s["part_w"][:, :, None] if c["weighted"] else a).sum(1)
    h = h.to(s["hidden"].dtype)
    f = h.float()
    y = f * torch.rsqrt(f.square().mean(1, keepdim=True) + EPS) * s["weight"].float()
    r = {"hidden": h}
    if c["out"]:
        r["out"] = y.to(h.dtype)
    if c["quant"]:
        scale = (y.abs().amax(1) / E4M3_MAX).clamp_min(TINY)
        r["quant"], r["scale"] = (y / scale[:, None]).to(DTYPE["e4m3"]), scale
    return r


def _plain_group(c, s):
    pick, G = s["pick"], c["groups"]
    key = torch.where((pick >= 0) & (pick < G), pick, G)
    order, at = torch.sort(key, stable=True)
    offsets = torch.searchsorted(order, torch.arange(G + 1, device="cuda", dtype=torch.int32))
    return {"rows": torch.where(order < G, at, -1).to(torch.int32),
            "offsets": offsets.to(torch.int32)}


def _plain_grouped(c, s):
    G, k, off = c["groups"], c["picks"], s["offsets"].long()
    src = s["rows"].long()
    m = src.numel()
    x = s["x"].float()
    if c["dtype"] == "e4m3":
        x = x * s["x_scale"][:, None]
    if c["gather"]:
        x = x[src // k]
    # every group's rows, padded to the longest group's
    at = torch.arange(m, device="cuda")
    g = torch.searchsorted(off, at, right=True) - 1
    slot = at - off[g]
    longest = int((off[1:] - off[:-1]).max())
    padded = x.new_zeros((G, longest, c["d_in"]))
    padded[g, slot] = x
    columns = padded.transpose(1, 2).contiguous()

    def product(name):
        w = s[name].float()
        if c["dtype"] == "e4m3":
            w = w * s[name + "_scale"][:, :, None]
        return torch.bmm(w, columns).transpose(1, 2)[g, slot]

    y = product("w")
    if c["swiglu"]:
        y = y / (1 + torch.exp(-y)) * product("w_up")
    if c["scatter"]:
        back = torch.empty_like(y)
        back[src] = y
        y = back
    return y.to(s["out"].dtype)


def _plain_quant(c, s):
    x = s["x"].float()

    def product(name):
        q = torch.stack([s[name] & 15, s[name] >> 4], 2).reshape(c["d_out"], -1, c["group"])
        zero = s[name + "_zero"][:, :, None].float() if c["zero"] else 8.0
        w = (q.float() - zero) * s[name + "_scale"][:, :, None].float()
        return x @ w.reshape(c["d_out"], c["d_in"]).T

    y = product("w")
    if c["swiglu"]:
        y = y / (1 + torch.exp(-y)) * product("up")
    if c["add"]:
        y = s["add"].float() + y
    return y.to(s["out"].dtype)


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------

def _own(c, s):
    from paper_2607_16305_amd import lookme as lk
    kind = c["kind"]
    if kind == "norm":
        lk.residual_norm(s["hidden"], weight=s["weight"], eps=EPS, add=s.get("add"),
                         part_w=s.get("part_w"), hidden_out=s["hidden_out"], out=s["out"],
                         out_quant=s["out_quant"], scale_out=s["scale_out"])
        r = {"hidden": s["hidden_out"]}
        if c["out"]:
            r["out"] = s["out"]
        if c["quant"]:
            r["quant"], r["scale"] = s["out_quant"], s["scale_out"]
        return r
    if kind == "group":
        lk.group_rows(s["pick"], c["groups"], s["rows_out"], s["offsets_out"])
        return {"rows": s["rows_out"], "offsets": s["offsets_out"]}
    if kind == "grouped":
        lk.grouped_product(s["x"], s["w"], s["offsets"], s["out"],
                           rows=s["rows"] if c["gather"] or c["scatter"] else None,
                           picks=c["picks"] if c["gather"] else 1, w_up=s.get("w_up"),
                           scatter=c["scatter"], x_scale=s.get("x_scale"),
                           w_scale=s.get("w_scale"), w_up_scale=s.get("w_up_scale"))
        return s["out"]
    if c["swiglu"]:
        lk.quant_swiglu(s["x"], s["w"], s["w_scale"], s["up"], s["up_scale"], s["out"],
                        z_gate=s.get("w_zero"), z_up=s.get("up_zero"))
    else:
        lk.quant_product(s["x"], s["w"], s["w_scale"], s["out"], zero=s.get("w_zero"),
                         add=s.get("add"))
    return s["out"]


def run(state):
    c = state["case"]
    if own:
        return _own(c, state)
    return {"norm": _plain_norm, "group": _plain_group, "grouped": _plain_grouped,
            "quant": _plain_quant}[c["kind"]](c, state)


# ---------------------------------------------------------------------------
# work and exact values
# ---------------------------------------------------------------------------

def _size(c):
    return {"bf16": 2, "f32": 4, "e4m3": 1}[c["dtype"]]


def work(case):
    c, kind = case, case["kind"]
    if kind == "norm":
        e, el = _size(c), c["n"] * c["d"]
        b = el * e * (2 + c["parts"]) + c["d"] * e + el * e * c["out"] + (el + 4 * c["n"]) * c["quant"]
        return {"bytes": b + 4 * c["n"] * c["parts"] * c["weighted"],
                "flops": el * (5 + 2 * c["parts"] + 2 * c["quant"])}
    if kind == "group":
        return {"bytes": 8 * c["n"] + 4 * (c["groups"] + 1), "flops": 0}
    if kind == "grouped":
        m, e = c["tokens"] * c["picks"], _size(c)
        mats = 2 if c["swiglu"] else 1
        # the weights of the groups that some token picks, of equal popularity
        used = c["groups"] * (1 - (1 - c["picks"] / c["groups"]) ** c["tokens"])
        w = used * mats * c["d_out"] * (c["d_in"] * e + (4 if e == 1 else 0))
        x = (c["tokens"] if c["gather"] else m) * (c["d_in"] * e + (4 if e == 1 else 0))
        out = m * c["d_out"] * (4 if c["dtype"] == "f32" else 2)
        index = 4 * (c["groups"] + 1) + (4 * m if c["gather"] or c["scatter"] else 0)
        return {"bytes": w + x + out + index, "flops": 2 * m * c["d_in"] * c["d_out"] * mats}
    e, mats = _size(c), 2 if c["swiglu"] else 1
    groups = c["d_in"] // c["group"]
    w = mats * c["d_out"] * (c["d_in"] // 2 + groups * (e + (1 if c["zero"] else 0)))
    return {"bytes": w + c["n"] * e * (c["d_in"] + c["d_out"] * (2 if c["add"] else 1)),
            "flops": 2 * c["n"] * c["d_in"] * c["d_out"] * mats}


def _silu64(v):
    return v / (1 + torch.exp(-v))


def exact(case, seed):
    c, s, kind = case, _inputs(case, seed), case["kind"]
    if kind == "group":
        return None
    if kind == "norm":
        total = s["hidden"].double()
        for j in range(c["parts"]):
            part = s["add"][:, j].double()
            total += part * s["part_w"][:, j:j + 1].double() if c["weighted"] else part
        f = total.to(s["hidden"].dtype).double()   # the sum is stored before it is normed
        y = f / torch.sqrt((f * f).mean(1, keepdim=True) + EPS) * s["weight"].double()
        r = {"hidden": total}
        if c["out"]:
            r["out"] = y
        if c["quant"]:
            r["scale"] = y.abs().amax(1) / E4M3_MAX
            r["quant"] = y / r["scale"][:, None].clamp_min(TINY)
        return r
    if kind == "grouped":
        off, rows = s["offsets"].tolist(), s["rows"].long()
        out = torch.zeros((rows.numel(), c["d_out"]), dtype=torch.float64, device="cuda")
        for g in range(c["groups"]):
            a, b = off[g], off[g + 1]
            if a == b:
                continue
            at = rows[a:b] // c["picks"] if c["gather"] else torch.arange(a, b, device="cuda")
            x = s["x"][at].double()
            if "x_scale" in s:
                x = x * s["x_scale"][at, None].double()
            ys = []
            for name in ("w", "w_up")[:2 if c["swiglu"] else 1]:
                w = s[name][g].double()
                if name + "_scale" in s:
                    w = w * s[name + "_scale"][g, :, None].double()
                ys.append(x @ w.T)
            y = _silu64(ys[0]) * ys[1] if c["swiglu"] else ys[0]
            out[rows[a:b] if c["scatter"] else slice(a, b)] = y
        return out
    ys = []
    for name in ("w", "up")[:2 if c["swiglu"] else 1]:
        w = torch.empty((c["d_out"], c["d_in"]), dtype=torch.float64, device="cuda")
        w[:, 0::2] = (s[name] & 15).double()
        w[:, 1::2] = (s[name] >> 4).double()
        each = lambda t: t.double().repeat_interleave(c["group"], 1)  # noqa: E731
        w -= each(s[name + "_zero"]) if c["zero"] else 8.0
        w *= each(s[name + "_scale"])
        ys.append(s["x"].double() @ w.T)
    y = _silu64(ys[0]) * ys[1] if c["swiglu"] else ys[0]
    return s["add"].double() + y if c["add"] else y
