"""The key/value cache in 8 bits: its operators as a program calls them, to be timed and compared.

A cache holds e4m3 codes [sequences, kv heads, capacity, head dim] for keys and values and one 32-bit
power-of-two scale per (sequence, kv head, block of tokens).  A case names an operator (``op``):

``append``  new tokens' keys and values are quantised and stored from position ``pos`` of each sequence on;
``attend``  query rows attend over a sequence's cached tokens and the call's own keys and values; with ``track``
            every cached token's softmax weights are added to its accumulated weight;
``evict``   of each (sequence, kv head) the ``keep`` tokens of the largest accumulated weight go to another cache.

The plain forms below are elementary tensor operations in 32 bits; ``exact`` repeats them in 64 bits from the
operators' definitions, sequence by sequence.
"""

import math

import torch

own = False
DEV = "cuda:0"

# heads as query / key-value x dim: those of this repository's experts, and two in between
HEADS = {"tiny": (4, 4, 32), "small": (8, 8, 64), "pi": (8, 1, 256), "large": (16, 4, 128), "mid": (8, 2, 128),
         "wide": (12, 3, 64)}


def _case(op, heads, **kw):
    nq, nkv, hd = HEADS[heads]
    c = dict(op=op, nq=nq, nkv=nkv, hd=hd, dtype="bf16", block=64, batch=1, pool=1, cap=64, n=1, fill=0, ragged=False,
             rows=1, self=0, track=False, keep=0, first=0)
    c.update(kw)
    return c


def listed():
    cases = {
        # one robot's step over its prefix of 816 tokens, two context slots, 50 buffer tokens: latency
        "attend_robot_b1": _case("attend", "pi", pool=2, cap=816, rows=50, self=50),
        # a fleet of 64 environments, the largest call of a rolling step
        "attend_fleet_b64": _case("attend", "pi", batch=64, pool=2, cap=816, rows=50, self=50),
        # the large expert, 16 environments whose prefixes have different lengths
        "attend_large_b16": _case("attend", "large", batch=16, cap=2048, rows=100, self=100, ragged=True),
        # the same call with the accumulated weights an eviction goes by
        "attend_track_b16": _case("attend", "pi", batch=16, cap=816, rows=50, self=50, track=True),
        # one new token of one sequence: serving's smallest call
        "attend_token_b1": _case("attend", "large", cap=4096, ragged=True),
        # one new token of each of 64 sequences of up to 16384 tokens: memory
        "attend_token_b64": _case("attend", "large", batch=64, cap=16384, ragged=True, block=128),
        # 32 bits, four small sequences, one of them empty
        "attend_small_f32": _case("attend", "small", batch=4, pool=2, cap=257, rows=16, self=16, ragged=True,
                                  dtype="f32", block=32),
        # one token's keys and values for each of 64 sequences, inside a block that older tokens fill
        "append_token_b64": _case("append", "large", batch=64, pool=2, cap=1024, n=1, fill=700),
        # a prefix of 18 layers published for one environment
        "append_context": _case("append", "pi", batch=18, pool=2, cap=816, n=816),
        # prompts of different lengths stored behind earlier tokens, in 32 bits as computed
        "append_prompts": _case("append", "large", batch=96, cap=4096, n=2000, fill=1001, ragged=True, dtype="f32"),
        # the 18 layers' prefix of one environment shortened to 256 tokens
        "evict_context": _case("evict", "pi", batch=18, cap=816, keep=256, first=4),
        # long sequences cut to a quarter
        "evict_long": _case("evict", "large", batch=32, cap=16384, keep=4096, first=4, ragged=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Any operator, heads, block and length from one token on, odd sizes more often than not; never more work than
    the largest listed case of the operator."""
    while True:
        op = rng.choice(["attend", "attend", "attend", "append", "evict"])
        c = _case(op, rng.choice(sorted(HEADS)), batch=_log_int(rng, 1, 64), pool=rng.randint(1, 3),
                  cap=_log_int(rng, 8, 16384), block=rng.choice([16, 32, 64, 64, 128]), ragged=rng.random() < 0.6,
                  dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        if op == "attend":
            c["rows"] = rng.choice([1, 1, _log_int(rng, 2, 128), _log_int(rng, 2, 128)])
            c["self"] = rng.choice([0, c["rows"], rng.randint(1, 128)])
            c["track"] = rng.random() < 0.3
        if op == "append":
            c["n"] = rng.choice([1, _log_int(rng, 1, c["cap"])])
            c["fill"] = rng.choice([0, rng.randint(0, c["cap"] - c["n"])])
        if op == "evict":
            c["keep"] = rng.randint(1, c["cap"])
            c["first"] = min(c["keep"], rng.choice([0, 1, 4]))
        tokens = c["batch"] * c["pool"] * c["cap"] * c["nkv"] * c["hd"]
        w = work(c)
        most = {"attend": 2.4e10, "append": 1e30, "evict": 1e30}[op] * (0.02 if c["dtype"] == "f32" else 1)
        if (w["flops"] <= most and tokens <= 64 * 16384 * 512 and
                w["bytes"] <= {"attend": 1e9, "append": 9e8, "evict": 4e8}[op]):
            return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _power(amax):
    """The smallest power of two, 2^-100 at least, by which amax (32 bits) divided is at most 448."""
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [1/2, 1); 448 = 0.875 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e, -100).clamp(min=-100))


def _code(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _quantised(x, block):
    """x [S, nkv, cap, hd] (32 bits) as codes and scales, blocks of tokens from position 0 on."""
    S, h, cap, hd = x.shape
    nb = -(-cap // block)
    pad = torch.nn.functional.pad(x, (0, 0, 0, nb * block - cap))
    s = _power(pad.view(S, h, nb, block * hd).abs().amax(-1))
    return _code(x / s.repeat_interleave(block, 2)[:, :, :cap, None]), s


def _lengths(c, g):
    """Cached tokens of each batch row: the capacity, or spread down to none."""
    B, cap = c["batch"], c["cap"]
    if not c["ragged"]:
        return torch.full((B,), cap, dtype=torch.int32, device=DEV)
    n = cap - (torch.rand(B, generator=g, device=DEV) * cap * 0.75).to(torch.int32)
    if B >= 4:
        n[1] = 0
    return n


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed * 2654435761 % (1 << 31) + 1)
    T = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    B, nkv, hd, cap, block = c["batch"], c["nkv"], c["hd"], c["cap"], c["block"]
    S = B * c["pool"]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=DEV, dtype=dtype)

    def tokens(*shape):  # keys and values as projections give them: channels of different size
        return normal(*shape, dtype=torch.bfloat16) * torch.exp(0.5 * normal(shape[-1])).to(torch.bfloat16)

    s = dict(case=c)
    kept = c["fill"] if c["op"] == "append" else cap  # tokens that are there before the call
    for x in ("k", "v"):
        codes = torch.zeros((S, nkv, cap, hd), dtype=torch.float8_e4m3fn, device=DEV)
        scale = torch.ones((S, nkv, -(-cap // block)), dtype=torch.float32, device=DEV)
        if kept:
            step = max(1, (1 << 28) // (nkv * kept * hd))
            for i in range(0, S, step):
                q, sc = _quantised(tokens(min(step, S - i), nkv, kept, hd).float(), block)
                codes[i:i + step, :, :kept] = q
                scale[i:i + step, :, :sc.shape[2]] = sc
        s[x + "_codes"], s[x + "_scale"] = codes, scale
    s["length"] = torch.zeros(S, dtype=torch.int32, device=DEV)
    seq = torch.randperm(S, generator=g, device=DEV)[:B].to(torch.int32)
    s["seq"] = seq
    if c["op"] == "append":
        s["k_new"], s["v_new"] = tokens(B, c["n"], nkv, hd).to(T), tokens(B, c["n"], nkv, hd).to(T)
        s["pos"] = torch.full((B,), c["fill"], dtype=torch.int32, device=DEV)
        s["count"] = torch.full((B,), c["n"], dtype=torch.int32, device=DEV)
        if c["ragged"]:
            s["pos"] -= (torch.rand(B, generator=g, device=DEV) * c["fill"] * 0.5).to(torch.int32)
            s["count"] -= (torch.rand(B, generator=g, device=DEV) * c["n"] * 0.75).to(torch.int32)
        s["length"][seq.long()] = c["fill"]
        return s
    s["length"][seq.long()] = _lengths(c, g)
    if c["op"] == "attend":
        s["q"] = normal(B, c["rows"], c["nq"], hd).to(T)
        s["k_self"] = s["v_self"] = None
        if c["self"]:
            s["k_self"], s["v_self"] = tokens(B, c["self"], nkv, hd).to(T), tokens(B, c["self"], nkv, hd).to(T)
        s["out"] = torch.empty_like(s["q"])
        if c["track"]:
            s["weight_before"] = torch.rand((S, nkv, cap), generator=g, device=DEV)
            s["weight"] = s["weight_before"].clone()
        return s
    # accumulated weights fall off fast; held to 7 bits here, so that some are equal
    s["weight"] = torch.exp(2.0 * normal(S, nkv, cap)).to(torch.bfloat16).float()
    room = c["keep"] + 5
    s["into"] = dict(k_codes=torch.zeros((B, nkv, room, hd), dtype=torch.float8_e4m3fn, device=DEV),
                     v_codes=torch.zeros((B, nkv, room, hd), dtype=torch.float8_e4m3fn, device=DEV),
                     k_scale=torch.ones((B, nkv, -(-room // block)), device=DEV),
                     v_scale=torch.ones((B, nkv, -(-room // block)), device=DEV),
                     length=torch.zeros(B, dtype=torch.int32, device=DEV), weight=torch.zeros((B, nkv, room), device=DEV))
    s["kept"] = torch.empty((B, nkv, c["keep"]), dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _bits(codes):
    return codes.view(torch.uint8)  # indexing and scattering of codes


def _store(c, codes, scale, new, seq, pos, count):
    B, n, nkv, hd = new.shape
    cap, block, nb = c["cap"], c["block"], scale.shape[2]
    wb = min(nb, (n + block - 2) // block + 1)  # blocks that n tokens can touch
    blk = (pos[:, None] // block + torch.arange(wb, device=DEV)).clamp(max=nb - 1)  # [B, wb]
    t = (blk[:, :, None] * block + torch.arange(block, device=DEV)).clamp(max=cap - 1)  # [B, wb, block]
    fresh = (t >= pos[:, None, None]) & (t < (pos + count)[:, None, None])
    old = t < pos[:, None, None]
    b = torch.arange(B, device=DEV)
    x = new.float()[b[:, None, None], (t - pos[:, None, None]).clamp(0, n - 1).long()]  # [B, wb, block, nkv, hd]
    was = _bits(codes).permute(0, 2, 1, 3)[seq[:, None, None], t.long()].view(torch.float8_e4m3fn).float()
    s0 = scale.permute(0, 2, 1)[seq[:, None], blk.long()]  # [B, wb, nkv]
    need = _power((x.abs().amax(-1) * fresh[..., None]).amax(2))
    s1 = torch.where(fresh.any(2)[..., None], torch.where(old.any(2)[..., None], torch.maximum(need, s0), need), s0)
    value = torch.where(fresh[..., None, None], _code(x / s1[:, :, None, :, None]).float(),
                        _code(was * (s0 / s1)[:, :, None, :, None]).float())
    value = torch.where((fresh | old)[..., None, None], value, was).to(torch.float8_e4m3fn)
    _bits(codes).permute(0, 2, 1, 3)[seq[:, None, None], t.long()] = _bits(value)
    scale.permute(0, 2, 1)[seq[:, None], blk.long()] = s1


def _append(s):
    c, seq = s["case"], s["seq"].long()
    _store(c, s["k_codes"], s["k_scale"], s["k_new"], seq, s["pos"], s["count"])
    _store(c, s["v_codes"], s["v_scale"], s["v_new"], seq, s["pos"], s["count"])
    s["length"][seq] = (s["pos"] + s["count"]).to(torch.int32)


def _values(codes, scale, seq, block):
    x = _bits(codes)[seq].view(torch.float8_e4m3fn).float()
    return x * scale[seq].repeat_interleave(block, 2)[:, :, :x.shape[2], None]


def _attend(s):
    c, seq = s["case"], s["seq"].long()
    B, T, nq, hd = s["q"].shape
    nkv, G = c["nkv"], c["nq"] // c["nkv"]
    q = s["q"].float().view(B, T, nkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, nkv, G * T, hd) / math.sqrt(hd)
    k = _values(s["k_codes"], s["k_scale"], seq, c["block"])
    score = q @ k.transpose(2, 3).contiguous()
    hidden = torch.arange(c["cap"], device=DEV) >= s["length"][seq][:, None]
    score = score.masked_fill(hidden[:, None, None], -math.inf)
    v = _values(s["v_codes"], s["v_scale"], seq, c["block"])
    if s["k_self"] is not None:
        ks, vs = (x.float().permute(0, 2, 1, 3).contiguous() for x in (s["k_self"], s["v_self"]))
        score = torch.cat([score, q @ ks.transpose(2, 3).contiguous()], -1)
        v = torch.cat([v, vs], 2)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = (p @ v).view(B, nkv, G, T, hd).permute(0, 3, 1, 2, 4).reshape(B, T, nq, hd)
    s["out"].copy_(o)
    if c["track"]:
        s["weight"][seq] += p[..., :c["cap"]].sum(2)


def _evict(s):
    c, seq, into = s["case"], s["seq"].long(), s["into"]
    B, nkv, cap, keep, block = c["batch"], c["nkv"], c["cap"], c["keep"], c["block"]
    n = s["length"][seq][:, None, None]
    w = s["weight"][seq]
    idx = torch.arange(cap, device=DEV).expand(B, nkv, cap)
    key = torch.where(idx < c["first"], torch.full_like(w, math.inf), w)
    key = torch.where(idx < n, key, torch.full_like(w, -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, idx)
    kept = (rank < keep) & (idx < n)
    moved = torch.sort(torch.where(kept & (idx >= keep), idx, torch.full_like(idx, cap)), dim=-1).values
    place, stay = idx[..., :keep], kept[..., :keep]
    live = place < n
    hole = ~stay & live
    at = (hole.cumsum(-1) - 1).clamp(min=0)
    src = torch.where(hole, moved.gather(-1, at), place)
    src = torch.where(live, src, torch.zeros_like(src))
    m = src.shape[-1]
    nb = -(-m // block)
    for x in ("k", "v"):
        q = _bits(s[x + "_codes"])[seq].gather(2, src[..., None].expand(-1, -1, -1, c["hd"])).view(torch.float8_e4m3fn)
        st = s[x + "_scale"][seq].gather(2, src // block)  # each token's scale where it was
        pad = torch.nn.functional.pad(torch.where(live, st, torch.zeros_like(st)), (0, nb * block - m))
        sn = pad.view(B, nkv, nb, block).amax(-1)
        div = torch.where(sn > 0, sn, torch.ones_like(sn)).repeat_interleave(block, 2)[..., :m]
        code = _bits(_code(q.float() * (st / div)[..., None]))
        old = _bits(into[x + "_codes"])[:, :, :m]
        old.copy_(torch.where(live[..., None], code, old))
        os = into[x + "_scale"][:, :, :nb]
        os.copy_(torch.where(sn > 0, sn, os))
    ow = into["weight"][:, :, :m]
    ow.copy_(torch.where(live, w.gather(-1, src), ow))
    into["length"].copy_(s["length"][seq].clamp(max=keep))
    s["kept"].fill_(-1)
    s["kept"][..., :m] = torch.where(live, src, torch.full_like(src, -1)).to(torch.int32)


def _handle(codes, weight=None):
    from paper_2609_34170_amd import ravel

    return lambda block: ravel.Cache(codes["k_codes"], codes["v_codes"], codes["k_scale"], codes["v_scale"],
                                     codes["length"], block, weight=weight)


def run(state):
    s, c = state, state["case"]
    if c["track"]:
        s["weight"].copy_(s["weight_before"])
    if own:
        if "cache" not in s:  # the handles that a program keeps
            s["cache"] = _handle(s, s.get("weight"))(c["block"])
            if c["op"] == "evict":
                s["into_cache"] = _handle(s["into"], s["into"]["weight"])(c["block"])
        if c["op"] == "append":
            s["cache"].append(s["k_new"], s["v_new"], seq=s["seq"], pos=s["pos"], count=s["count"])
        elif c["op"] == "attend":
            s["cache"].attention(s["q"], s["out"], s["k_self"], s["v_self"], seq=s["seq"], track=c["track"])
        else:
            s["cache"].evict(c["keep"], first=c["first"], seq=s["seq"], into=s["into_cache"], kept=s["kept"])
    else:
        {"append": _append, "attend": _attend, "evict": _evict}[c["op"]](s)
    if c["op"] == "append":
        return {x: s[x] for x in ("k_codes", "k_scale", "v_codes", "v_scale", "length")}
    if c["op"] == "attend":
        return {"out": s["out"], "weight": s["weight"]} if c["track"] else s["out"]
    return {"kept": s["kept"], **s["into"]}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    """Codes count a byte, ragged lengths and counts their mean, scales and lengths their bytes."""
    c = case
    elt = 4 if c["dtype"] == "f32" else 2
    B, row = c["batch"], c["nkv"] * c["hd"]
    if c["op"] == "append":
        n = c["n"] * (0.625 if c["ragged"] else 1.0)
        return {"bytes": 2.0 * B * (n * row * (elt + 1) + c["nkv"] * (n / c["block"] + 1) * 4), "flops": 2.0 * B * n * row * 2}
    n = c["cap"] * (0.625 if c["ragged"] else 1.0)
    if c["op"] == "attend":
        keys = n + c["self"]
        data = 2.0 * B * (n * row + c["nkv"] * n / c["block"] * 4 + c["self"] * row * elt + c["rows"] * c["nq"] * c["hd"] * elt)
        if c["track"]:
            data += 8.0 * B * c["nkv"] * n
        return {"bytes": data, "flops": 4.0 * B * c["rows"] * c["nq"] * c["hd"] * keys}
    keep = min(n, c["keep"])
    return {"bytes": B * c["nkv"] * (4.0 * n + keep * (4 * c["hd"] + 4 + 4) + 16.0 * keep / c["block"]), "flops": 4.0 * B * c["nkv"] * keep * c["hd"]}


def _near(x):
    """The e4m3 number nearest to x (64 bits), halves to even."""
    a = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.round(a / step) * step * torch.sign(x)


def _scale64(amax):
    """Smallest power of two with amax / scale <= 448, 2^-100 at least; amax one 64-bit number a row."""
    e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448.0))
    e = torch.where(torch.exp2(e) * 448.0 < amax, e + 1, e)  # the logarithm's own rounding
    e = torch.where(torch.exp2(e - 1) * 448.0 >= amax, e - 1, e)
    return torch.exp2(e.clamp(min=-100))


def _exact_append(c, s):
    res = {"length": s["length"].clone()}
    for x in ("k", "v"):
        codes, scale = s[x + "_codes"].double(), s[x + "_scale"].double()
        for b, (q, p, m) in enumerate(zip(s["seq"].tolist(), s["pos"].tolist(), s["count"].tolist())):
            res["length"][q] = p + m
            new = s[x + "_new"][b, :m].double().permute(1, 0, 2)  # [nkv, m, hd]
            for blk in range(p // c["block"], (p + m - 1) // c["block"] + 1 if m else 0):
                lo, hi = max(p, blk * c["block"]), min(p + m, (blk + 1) * c["block"])
                to = _scale64(new[:, lo - p:hi - p].abs().amax((1, 2)))
                old = codes[q, :, blk * c["block"]:lo]
                if lo > blk * c["block"]:
                    to = torch.maximum(to, scale[q, :, blk])
                    codes[q, :, blk * c["block"]:lo] = _near(old * (scale[q, :, blk] / to)[:, None, None])
                codes[q, :, lo:hi] = _near(new[:, lo - p:hi - p] / to[:, None, None])
                scale[q, :, blk] = to
        res[x + "_codes"], res[x + "_scale"] = codes, scale
    return {x: res[x] for x in ("k_codes", "k_scale", "v_codes", "v_scale", "length")}


def _exact_attend(c, s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    weight = s["weight_before"].double() if c["track"] else None
    G = c["nq"] // c["nkv"]
    for b, q in enumerate(s["seq"].tolist()):
        n = int(s["length"][q])
        for h in range(c["nkv"]):
            at = torch.arange(n, device=DEV) // c["block"]
            k, v = (s[x + "_codes"][q, h, :n].double() * s[x + "_scale"][q, h].double()[at][:, None] for x in ("k", "v"))
            if s["k_self"] is not None:
                k, v = torch.cat([k, s["k_self"][b, :, h].double()]), torch.cat([v, s["v_self"][b, :, h].double()])
            if not len(k):
                continue
            rows = s["q"][b, :, h * G:(h + 1) * G].double().reshape(-1, c["hd"])
            p = torch.softmax(rows @ k.T / math.sqrt(c["hd"]), -1)
            out[b, :, h * G:(h + 1) * G] = (p @ v).view(-1, G, c["hd"])
            if c["track"]:
                weight[q, h, :n] += p[:, :n].sum(0)
    return {"out": out, "weight": weight} if c["track"] else out


def _exact_evict(c, s):
    into, keep = {x: t.double() if t.is_floating_point() else t.clone() for x, t in s["into"].items()}, c["keep"]
    kept = torch.full(s["kept"].shape, -1, dtype=torch.int64)
    for b, q in enumerate(s["seq"].tolist()):
        n = int(s["length"][q])
        m = min(n, keep)
        into["length"][b] = m
        for h in range(c["nkv"]):
            w = s["weight"][q, h, :n].double().cpu()
            w[:c["first"]] = math.inf
            best = torch.sort(w, descending=True, stable=True).indices[:m]
            inside, outside = best[best < m], torch.sort(best[best >= m]).values
            src = torch.full((m,), -1, dtype=torch.int64)
            src[inside] = inside
            src[src < 0] = outside
            kept[b, h, :m] = src
            src = src.to(DEV)
            into["weight"][b, h, :m] = s["weight"][q, h][src].double()
            for x in ("k", "v"):
                sc = s[x + "_scale"][q, h].double()[src // c["block"]]
                blocks = torch.arange(m, device=DEV) // c["block"]
                top = torch.zeros(-(-m // c["block"]), dtype=torch.float64, device=DEV).scatter_reduce(0, blocks, sc, "amax")
                into[x + "_codes"][b, h, :m] = _near(s[x + "_codes"][q, h][src].double() * (sc / top[blocks])[:, None])
                into[x + "_scale"][b, h, :len(top)] = top
    return {"kept": kept, **into}


def exact(case, seed):
    c = case
    if c["op"] != "attend" and c["batch"] * c["pool"] * c["cap"] * c["nkv"] * c["hd"] > 1 << 27:
        return None  # the results alone take minutes to form block by block
    s = prepare(c, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[c["op"]](c, s)
