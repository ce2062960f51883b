"""A layer's operators for training and serving, as a program calls them between its linear layers, to be timed and
compared.

A case names an operator (``op``); ``train`` adds its gradients to the pass.

``norm``    gated residual and norm: t = x + alpha * gate * F with F = f or rms(f) (1 + post), y = rms(t) (1 + scale) +
            shift.  Modulation rows are one per row, per group of rows or per place in a period, or one vector;
``attend``  cross attention of query rows to an encoder's states of another length, grouped heads;
``mlp``     gated MLP up to its hidden values: h = act(x Wg^T) * (x Wu^T).

The plain forms below are elementary tensor operations in 32 bits with the gradients written out; ``exact`` gets them in
64 bits from the forward definitions by automatic differentiation.
"""

import math

import torch

own = False
DEV = "cuda:0"

# heads as query / key-value x dim, width and hidden size: those of this repository's experts, and some in between
HEADS = {"tiny": (4, 4, 32), "small": (8, 8, 64), "pi": (8, 1, 256), "large": (16, 4, 128), "mid": (8, 2, 128),
         "wide": (12, 3, 64)}
MLPS = {"tiny": (128, 512), "small": (512, 2048), "pi": (1024, 4096), "large": (2048, 8192), "odd": (328, 888),
        "thin": (1000, 136)}


def _norm(rows, width, **kw):
    c = dict(op="norm", train=False, rows=rows, width=width, stream="f32", dtype="bf16", mods=rows, group=1, f=True,
             post=False, alpha=False, gate=True, static=False, shift=True)
    c.update(kw)
    return c


def _attend(heads, **kw):
    nq, nkv, hd = HEADS[heads]
    c = dict(op="attend", train=False, nq=nq, nkv=nkv, hd=hd, dtype="bf16", batch=1, rows=1, keys=16, ragged=False)
    c.update(kw)
    return c


def _mlp(size, **kw):
    w, hidden = MLPS[size]
    c = dict(op="mlp", train=False, rows=1, width=w, hidden=hidden, dtype="bf16", act="gelu")
    c.update(kw)
    return c


def listed():
    cases = {
        # between two blocks of one robot's step: 50 buffer rows, each with its own modulation
        "norm_step_b1": _norm(50, 1024),
        # a training batch of 64 samples, 50 rows each, modulated row by row
        "norm_fleet_train": _norm(3200, 1024, train=True),
        # adapters of the large expert: a normed block output under one scalar, vectors for all of 6400 rows
        "norm_adapter_train": _norm(6400, 2048, train=True, mods=1, post=True, alpha=True, gate=False, static=True,
                                    shift=False),
        # one query row of each of 64 sequences over encoder states of up to 4096 tokens: memory
        "attend_token_b64": _attend("large", batch=64, keys=4096, ragged=True),
        # adapters of 64 samples: 50 rows over 16 pathway tokens
        "attend_fop_train": _attend("pi", train=True, batch=64, rows=50, keys=16),
        # 16 contexts of up to 2048 tokens, eight horizons of 100 rows each: matrix products
        "attend_context_train": _attend("large", train=True, batch=16, rows=800, keys=2048, ragged=True),
        # 32 bits, small sequences of different lengths, one without keys
        "attend_small_f32_train": _attend("small", train=True, batch=8, rows=33, keys=257, ragged=True, dtype="f32"),
        # one token of the large expert: its weights are read once
        "mlp_token_b1": _mlp("large"),
        # one robot's step
        "mlp_step_b1": _mlp("pi", rows=50),
        # a training batch of 64 samples of 50 rows
        "mlp_fleet_train": _mlp("pi", train=True, rows=3200),
        # the large expert's, 64 samples of 100 rows: the largest products
        "mlp_large_train": _mlp("large", train=True, rows=6400),
        # 32 bits, sizes that no tile divides
        "mlp_odd_f32_train": _mlp("odd", train=True, rows=77, dtype="f32", act="silu"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Any operator, forward or with gradients, sizes from one row on, odd ones more often than not; never more work
    than the largest listed case of the operator."""
    while True:
        op = rng.choice(["norm", "attend", "mlp"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        train = rng.random() < 0.6
        if op == "norm":
            rows = _log_int(rng, 1, 20000)
            width = rng.choice([128, 512, 1024, 2048, 8 * _log_int(rng, 1, 1024)])
            kind = rng.choice(["row", "group", "period", "vector"])
            group, mods = {"row": (1, rows), "group": (_log_int(rng, 1, rows), 0), "period": (1, _log_int(rng, 1, rows)),
                           "vector": (1, 1)}[kind]
            mods = mods or -(-rows // group)
            c = _norm(rows, width, train=train, dtype=dtype, stream="f32" if dtype == "f32" else rng.choice(["f32", "bf16"]),
                      mods=mods, group=group, f=rng.random() < 0.8, static=rng.random() < 0.3, shift=rng.random() < 0.6)
            if c["f"]:
                c.update(post=rng.random() < 0.3, alpha=rng.random() < 0.3, gate=rng.random() < 0.7)
            else:
                c["gate"] = False
            most = dict(bytes=5e8, flops=1e30)
        elif op == "attend":
            c = _attend(rng.choice(sorted(HEADS)), train=train, dtype=dtype, batch=_log_int(rng, 1, 64),
                        rows=rng.choice([1, _log_int(rng, 1, 1000), _log_int(rng, 1, 1000)]), keys=_log_int(rng, 1, 8192),
                        ragged=rng.random() < 0.5)
            most = dict(bytes=7e8, flops=4e11 if dtype == "bf16" else 2e10)
        else:
            c = _mlp("tiny", train=train, dtype=dtype, rows=rng.choice([1, _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)]),
                     act=rng.choice(["gelu", "silu"]))
            c["width"], c["hidden"] = rng.choice(list(MLPS.values()) + [(8 * _log_int(rng, 1, 256), 8 * _log_int(rng, 1, 1024))])
            most = dict(bytes=1e9, flops=1.2e12 if dtype == "bf16" else 5e10)
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed * 2654435761 % (1 << 31) + 7)
    T = _type(c["dtype"])

    def normal(*shape, dtype=torch.float32, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)

    s = dict(case=c)
    if c["op"] == "norm":
        rows, w, mods, S = c["rows"], c["width"], c["mods"], _type(c["stream"])
        s["x"] = normal(rows, w, dtype=S) * 2
        if c["f"]:
            s["f"] = normal(rows, w, dtype=T)
            if c["post"]:
                s["post"] = normal(w, std=0.1)
            if c["alpha"]:
                s["alpha"] = normal(1, std=0.5)
            if c["gate"]:
                s["gate"] = normal(mods, w, std=0.3)
        # vectors, or the chunks of a conditioning layer's rows
        s["scale"] = normal(w, std=0.1) if c["static"] else normal(mods, 3 * w, std=0.2)[:, :w]
        if c["shift"]:
            s["shift"] = normal(w, std=0.1) if c["static"] else normal(mods, 3 * w, std=0.2)[:, w:2 * w]
        s["y"] = torch.empty((rows, w), dtype=T, device=DEV)
        s["x_out"] = torch.empty_like(s["x"]) if c["f"] else None
        if c["train"]:
            s["dy"], s["d_out"] = normal(rows, w, dtype=T), normal(rows, w, dtype=S)
            s["grads"] = {"x": torch.empty_like(s["x"])}
            if c["f"]:
                s["grads"]["f"] = torch.empty_like(s["f"])
            for x in ("post", "alpha", "gate", "scale", "shift"):
                if x in s:
                    s["grads"][x] = torch.empty(s[x].shape, device=DEV)
    elif c["op"] == "attend":
        B, nq, nkv, hd, R, K = (c[x] for x in ("batch", "nq", "nkv", "hd", "rows", "keys"))
        s["q"] = normal(B, R, nq, hd, dtype=T)
        # keys and values as one projection gives them: each token's key, then its value
        kv = (normal(B, K, 2, nkv, hd) * torch.exp(0.3 * normal(hd))).to(T)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["k_len"] = None
        if c["ragged"]:
            n = K - (torch.rand(B, generator=g, device=DEV) * K * 0.75).to(torch.int32)
            if B >= 4:
                n[1] = 0
            s["k_len"] = n.to(torch.int32)
        s["out"] = torch.empty_like(s["q"])
        if c["train"]:
            s["dout"] = normal(B, R, nq, hd, dtype=T)
            s["lse"] = torch.empty((B, nq, R), dtype=torch.float32, device=DEV)
            dkv = torch.empty_like(kv)
            s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), dkv[:, :, 0], dkv[:, :, 1]
    else:
        M, w, hidden = c["rows"], c["width"], c["hidden"]
        s["x"] = normal(M, w, dtype=T)
        s["wg"], s["wu"] = normal(hidden, w, dtype=T, std=0.02), normal(hidden, w, dtype=T, std=0.02)
        s["h"] = torch.empty((M, hidden), dtype=T, device=DEV)
        if c["train"]:
            s["dh"] = normal(M, hidden, dtype=T, std=0.1)
            s["g"], s["u"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
            s["dx"], s["dwg"], s["dwu"] = (torch.empty_like(s[x]) for x in ("x", "wg", "wu"))
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _rms(x, eps=1e-6):
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r


def _plain_norm(s):
    c = s["case"]
    rows, mods = c["rows"], c["mods"]
    at = (torch.arange(rows, device=DEV) // c["group"]) % mods

    def spread(t):  # a modulation for every row
        return t if t.dim() == 1 else t[at]

    def gather(d, like):  # a gradient of every row, summed over the rows that share the modulation
        if like.dim() == 1:
            return d.sum(0)
        return d if mods == rows and c["group"] == 1 else torch.zeros((mods, d.shape[1]), device=DEV).index_add_(0, at, d)

    t = s["x"].float()
    if c["f"]:
        f = s["f"].float()
        m, rf = _rms(f) if c["post"] else (f, None)
        F = m * (1 + s["post"]) if c["post"] else m
        ag = spread(s["gate"]) if c["gate"] else torch.ones((), device=DEV)
        if c["alpha"]:
            ag = ag * s["alpha"]
        t = (t + ag * F).to(s["x"].dtype).float()
    n, r = _rms(t)
    scale = 1 + spread(s["scale"])
    y = n * scale + spread(s["shift"]) if c["shift"] else n * scale
    res = {"y": y.to(s["y"].dtype)}
    if c["f"]:
        res["x_out"] = t.to(s["x"].dtype)
    if not c["train"]:
        return res
    dy, g = s["dy"].float(), {}
    dn = dy * scale
    dt = s["d_out"].float() + r * (dn - n * (dn * n).mean(-1, keepdim=True))
    g["x"] = dt.to(s["x"].dtype)
    g["scale"] = gather(dy * n, s["scale"])
    if c["shift"]:
        g["shift"] = gather(dy, s["shift"])
    if c["f"]:
        dF = dt * ag
        if c["gate"]:
            d = dt * F
            if c["alpha"]:
                g["alpha"] = (d * spread(s["gate"])).sum().view(1)
                d = d * s["alpha"]
            g["gate"] = gather(d, s["gate"])
        elif c["alpha"]:
            g["alpha"] = (dt * F).sum().view(1)
        if c["post"]:
            g["post"] = (dF * m).sum(0)
            dm = dF * (1 + s["post"])
            dF = rf * (dm - m * (dm * m).mean(-1, keepdim=True))
        g["f"] = dF.to(s["f"].dtype)
    return {**res, **{"d" + x: t for x, t in g.items()}}


def _plain_attend(s):
    c = s["case"]
    B, R, nq, hd = s["q"].shape
    nkv, K, G = c["nkv"], c["keys"], c["nq"] // c["nkv"]
    T, scale = s["q"].dtype, 1 / math.sqrt(hd)

    def rows(t):  # [B, nkv, G R, hd]
        return t.float().view(B, R, nkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, nkv, G * R, hd)

    def back(t):
        return t.view(B, nkv, G, R, hd).permute(0, 3, 1, 2, 4).reshape(B, R, nq, hd).to(T)

    q, k, v = rows(s["q"]), s["k"].float().permute(0, 2, 1, 3).contiguous(), s["v"].float().permute(0, 2, 1, 3).contiguous()
    score = q @ k.transpose(2, 3).contiguous() * scale
    if s["k_len"] is not None:
        hidden = torch.arange(K, device=DEV) >= s["k_len"][:, None]
        score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    del score
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = p @ v
    if not c["train"]:
        return {"out": back(o)}
    do = rows(s["dout"])
    dv = p.transpose(2, 3).contiguous() @ do
    ds = p * (do @ v.transpose(2, 3).contiguous() - (do * o).sum(-1, keepdim=True)) * scale
    dq, dk = ds @ k, ds.transpose(2, 3).contiguous() @ q
    return {"out": back(o), "dq": back(dq), "dk": dk.permute(0, 2, 1, 3).to(T), "dv": dv.permute(0, 2, 1, 3).to(T)}


def _act(g, kind):
    """Activation and its derivative."""
    if kind == "silu":
        y = 1 / (1 + torch.exp(-g))
        return g * y, y * (1 + g * (1 - y))
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * 0.044715 * g * g)


def _plain_mlp(s):
    c, T = s["case"], s["x"].dtype
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _act(g, c["act"])
    res = {"h": (a * u).to(T)}
    if not c["train"]:
        return res
    dh = s["dh"].float()
    dg, du = dh * u * slope, dh * a
    return {**res, "dx": (dg @ wg + du @ wu).to(T), "dwg": (dg.t() @ x).to(T), "dwu": (du.t() @ x).to(T)}


def _own(s):
    from paper_2609_34170_amd import ravel

    c = s["case"]
    if c["op"] == "norm":
        mod = {x: s.get(x) for x in ("f", "post", "alpha", "gate", "scale")}
        ravel.norm_residual(s["x"], **mod, shift=s.get("shift"), group=c["group"], y=s["y"], x_out=s["x_out"])
        res = {"y": s["y"]}
        if c["f"]:
            res["x_out"] = s["x_out"]
        if c["train"]:
            ravel.norm_residual_grad(s["x_out"] if c["f"] else s["x"], s["dy"], s["d_out"], **mod, group=c["group"],
                                     grads=s["grads"])
            res.update({"d" + x: t for x, t in s["grads"].items()})
        return res
    if c["op"] == "attend":
        ravel.cross_attention(s["q"], s["k"], s["v"], k_len=s["k_len"], out=s["out"], lse=s.get("lse"))
        if not c["train"]:
            return {"out": s["out"]}
        ravel.cross_attention_grad(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], k_len=s["k_len"], dq=s["dq"],
                                   dk=s["dk"], dv=s["dv"])
        return {x: s[x] for x in ("out", "dq", "dk", "dv")}
    if not c["train"]:
        ravel.gated_mlp(s["x"], s["wg"], s["wu"], act=c["act"], h=s["h"])
        return {"h": s["h"]}
    # what the gradients go on from stays in 32 bits, as in the plain form, in memory that a program keeps as it keeps h's
    if s["g"].dtype is not torch.float32:
        s["g"], s["u"] = (torch.empty(t.shape, device=DEV) for t in (s["g"], s["u"]))
    gate, up = s["g"], s["u"]
    ravel.gated_mlp(s["x"], s["wg"], s["wu"], act=c["act"], h=s["h"], gate=gate, up=up)
    ravel.gated_mlp_grad(s["x"], s["wg"], s["wu"], gate, up, s["dh"], act=c["act"], dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"])
    return {x: s[x] for x in ("h", "dx", "dwg", "dwu")}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "attend": _plain_attend, "mlp": _plain_mlp}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    """Each input once, each output once; lengths that differ count their mean.  What a forward leaves for its gradients
    (lse, gate and up values) and reading anything a second time are not counted."""
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "norm":
        S, rows, w = 4 if c["stream"] == "f32" else 2, c["rows"], c["width"]
        vec = w if c["static"] else c["mods"] * w
        mod = 4.0 * (vec * (2 if c["shift"] else 1) + (c["mods"] * w if c["gate"] else 0) + (w if c["post"] else 0))
        data = rows * w * (S + e + (S + e if c["f"] else 0)) + mod
        if c["train"]:
            data += rows * w * (e + S + S + (e if c["f"] else 0)) + mod
        return {"bytes": float(data), "flops": float(rows * w * (40 if c["train"] else 10))}
    if c["op"] == "attend":
        n = c["keys"] * (0.625 if c["ragged"] else 1.0)
        data = c["batch"] * e * (2.0 * c["rows"] * c["nq"] * c["hd"] + 2 * n * c["nkv"] * c["hd"])
        pair = 2.0 * c["batch"] * c["rows"] * c["nq"] * c["hd"] * n
        if c["train"]:
            data += c["batch"] * e * (2.0 * c["rows"] * c["nq"] * c["hd"] + 2 * c["keys"] * c["nkv"] * c["hd"])
        return {"bytes": data, "flops": pair * (7 if c["train"] else 2)}
    M, w, hidden = c["rows"], c["width"], c["hidden"]
    data = e * (M * w + M * hidden + 2.0 * w * hidden)
    if c["train"]:
        data += e * (M * hidden + M * w + 2.0 * w * hidden)
    return {"bytes": float(data), "flops": (12.0 if c["train"] else 4.0) * M * w * hidden}


def _leaf(t):
    return t.double().clone().requires_grad_()


def _exact_norm(c, s):
    at = (torch.arange(c["rows"], device=DEV) // c["group"]) % c["mods"]
    x = {n: _leaf(s[n]) for n in ("x", "f", "post", "alpha", "gate", "scale", "shift") if n in s}

    def of_rows(t):
        return t if t.dim() == 1 else t.index_select(0, at)

    def unit(t):
        return t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6)

    t = x["x"]
    if c["f"]:
        b = unit(x["f"]) * (x["post"] + 1) if c["post"] else x["f"]
        b = b * of_rows(x["gate"]) if c["gate"] else b
        t = t + (b * x["alpha"] if c["alpha"] else b)
    # a 16-bit residual stream is what it is rounded to, for the norm behind it as well
    held = t if c["stream"] == "f32" else t + (t.to(torch.bfloat16).double() - t).detach()
    y = unit(held) * (of_rows(x["scale"]) + 1)
    if c["shift"]:
        y = y + of_rows(x["shift"])
    res = {"y": y.detach()}
    if c["f"]:
        res["x_out"] = held.detach()
    if c["train"]:
        names = [n for n in ("x", "scale", "shift", "alpha", "gate", "post", "f") if n in x]
        d = torch.autograd.grad([y, held], [x[n] for n in names], [s["dy"].double(), s["d_out"].double()])
        res.update({"d" + n: g for n, g in zip(names, d)})
    return res


def _exact_attend(c, s):
    G = c["nq"] // c["nkv"]
    res = {n: torch.zeros(s[m].shape, dtype=torch.float64, device=DEV)
           for n, m in (("out", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    for b in range(c["batch"]):
        n = c["keys"] if s["k_len"] is None else int(s["k_len"][b])
        if n == 0:
            continue
        for h in range(c["nkv"]):
            q, k, v = _leaf(s["q"][b, :, h * G:(h + 1) * G]), _leaf(s["k"][b, :n, h]), _leaf(s["v"][b, :n, h])
            o = torch.softmax(q.reshape(-1, c["hd"]) @ k.T / math.sqrt(c["hd"]), -1) @ v
            o = o.view(q.shape)
            res["out"][b, :, h * G:(h + 1) * G] = o.detach()
            if c["train"]:
                dq, dk, dv = torch.autograd.grad(o, [q, k, v], s["dout"][b, :, h * G:(h + 1) * G].double())
                res["dq"][b, :, h * G:(h + 1) * G], res["dk"][b, :n, h], res["dv"][b, :n, h] = dq, dk, dv
    return res if c["train"] else {"out": res["out"]}


def _exact_mlp(c, s):
    x, wg, wu = _leaf(s["x"]), _leaf(s["wg"]), _leaf(s["wu"])
    g, u = torch.nn.functional.linear(x, wg), torch.nn.functional.linear(x, wu)
    h = (torch.nn.functional.silu(g) if c["act"] == "silu" else torch.nn.functional.gelu(g, approximate="tanh")) * u
    if not c["train"]:
        return {"h": h.detach()}
    d = torch.autograd.grad(h, [x, wg, wu], s["dh"].double())
    return {"h": h.detach(), "dx": d[0], "dwg": d[1], "dwu": d[2]}


def exact(case, seed):
    return {"norm": _exact_norm, "attend": _exact_attend, "mlp": _exact_mlp}[case["op"]](case, prepare(case, seed))
