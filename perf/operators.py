"""Cases that stand for what a program has the language operators do: a decoder that answers over
frames, next to the CNN front-end whose feature maps it reads.

A feature map in NHWC is a sequence of H * W states per frame: 196 at 224 pixels, 676 at 416,
1444 at 608 and 5776 at 1216.  Three operators read them or what comes of them:

``norm``    h = x + r; y = h / sqrt(mean(h^2) + eps) * w, y in the inputs' type or in 8 bits (e4m3)
            with scales, one for a row or one for each 128 channels
``cross``   attention of n_q tokens to the n_kv states of their frame, some of them not readable
            (shorter maps, maps padded to a common size)
``prefix``  attention of requests in groups that share a prefix (a frame's states), each request
            with keys of its own behind it, for the last n_q tokens of the request

Inputs are normal; projections of normalised states have unit variance.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
E4M3_MAX = 448.0


def _norm(name, rows, cols, dtype, quant, residual=True):
    # quant: "none", "row" (one scale a row) or "128" (one scale for each 128 channels)
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "quant": quant, "residual": residual}


def _cross(name, batch, n_q, n_kv, heads_q, heads_kv, dim, dtype, lengths="full"):
    # lengths: "full"; "ragged" (each sequence has a length of its own); "padded" (each map is a
    # rectangle inside the padded one: a mask)
    return {"name": name, "op": "cross", "batch": batch, "n_q": n_q, "n_kv": n_kv, "heads_q": heads_q,
            "heads_kv": heads_kv, "dim": dim, "dtype": dtype, "lengths": lengths}


def _prefix(name, prefixes, requests, n_q, n_prefix, n_own, heads_q, heads_kv, dim, dtype):
    return {"name": name, "op": "prefix", "prefixes": prefixes, "requests": requests, "n_q": n_q, "n_prefix": n_prefix,
            "n_own": n_own, "heads_q": heads_q, "heads_kv": heads_kv, "dim": dim, "dtype": dtype}


def listed():
    return [
        # one decoding step of 16 requests before an 8-bit projection: latency
        _norm("norm_step_16x1024", 16, 1024, "bf16", "row"),
        # the states of sixteen 608x608 frames, normalised before they are projected
        _norm("norm_b16_608_256", 16 * 1444, 256, "bf16", "none"),
        # eight frames at 1216 pixels in 1024 channels, in 8 bits by blocks of channels
        _norm("norm_b8_1216_1024", 8 * 5776, 1024, "bf16", "128"),
        # odd sizes in single precision
        _norm("norm_fp32_1443x1001", 1443, 1001, "fp32", "none"),
        # the smallest attention call: one token of one request looks at a 608x608 frame
        _cross("cross_token_608", 1, 1, 1444, 8, 4, 64, "bf16"),
        # a server's decoding step: 64 requests, each with a frame of its own size
        _cross("cross_step_b64_608", 64, 1, 1444, 32, 8, 128, "bf16", "ragged"),
        # prompts of odd length over four frames, every head with its own keys
        _cross("cross_prompt_333_608", 4, 333, 1444, 16, 16, 64, "bf16"),
        # the largest: long texts over eight frames of different shapes at 1216 pixels
        _cross("cross_long_b8_1216", 8, 2048, 5776, 16, 4, 128, "bf16", "padded"),
        # single precision: short texts over 416x416 frames
        _cross("cross_fp32_77_416", 2, 77, 676, 8, 2, 128, "fp32", "ragged"),
        # a decoding step of 16 questions about one 608x608 frame
        _prefix("prefix_step_608_r16", 1, 16, 1, 1444, 96, 16, 4, 64, "bf16"),
        # a decoding step of 64 requests about a clip of sixteen 608x608 frames
        _prefix("prefix_step_clip_r64", 1, 64, 1, 16 * 1444, 512, 32, 8, 128, "bf16"),
        # the prompts of eight requests about each of four frames at 1216 pixels
        _prefix("prefix_prompt_1216_4x8", 4, 8, 61, 5776, 200, 16, 4, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "cross", "cross", "cross", "prefix", "prefix", "prefix"])
    if op == "norm":
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        cols = rng.choice([_log_int(rng, 64, 4096), 8 * _log_int(rng, 8, 1024)])
        rows = min(_log_int(rng, 1, 50000), max(1, 46_000_000 // cols))
        c = _norm("", rows, cols, dtype, rng.choice(["none", "row", "128"]), rng.random() < 0.8)
    else:
        dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "fp32"])
        dim = rng.choice([64, 64, 128, 128, 80, 40])
        heads_kv = rng.choice([1, 2, 4, 8])
        heads_q = heads_kv * rng.choice([1, 2, 4, 8])
        # pairs of a query and a key, and elements of k and v: within the largest listed case
        pairs = (250_000_000 if dtype == "fp32" else 1_200_000_000) // heads_q
        keys = 90_000_000 // (heads_kv * dim)
        if op == "cross":
            n_kv = min(_log_int(rng, 1, 6000), keys)
            n_q = 1 if rng.random() < 0.4 else min(_log_int(rng, 2, 2048), max(1, pairs // n_kv))
            batch = max(1, min(_log_int(rng, 1, 64), pairs // (n_q * n_kv), keys // n_kv))
            c = _cross("", batch, n_q, n_kv, heads_q, heads_kv, dim, dtype, rng.choice(["full", "ragged", "padded"]))
        else:
            n_prefix = min(_log_int(rng, 16, 24000), keys // 2)
            n_own = _log_int(rng, 1, 600)
            n_q = 1 if rng.random() < 0.6 else rng.randint(2, min(96, n_own + 1))
            n_own = max(n_own, n_q)
            both = n_prefix + n_own
            prefixes = max(1, min(_log_int(rng, 1, 8), keys // (2 * n_prefix), pairs // (n_q * both)))
            requests = max(1, min(_log_int(rng, 1, 64), keys // (2 * n_own * prefixes), pairs // (n_q * both * prefixes)))
            c = _prefix("", prefixes, requests, n_q, n_prefix, n_own, heads_q, heads_kv, dim, dtype)
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------


def _mask(g, batch, n_kv):
    """Readable places of maps padded to one size: a rectangle of each map's own size in the corner
    of the common one, whose width is about the root of n_kv."""
    w = max(1, math.isqrt(n_kv))
    h = -(-n_kv // w)
    own_h = torch.randint((h + 1) // 2, h + 1, (batch, 1), generator=g, device="cuda")
    own_w = torch.randint((w + 1) // 2, w + 1, (batch, 1), generator=g, device="cuda")
    at = torch.arange(n_kv, device="cuda")[None]
    return (at // w < own_h) & (at % w < own_w)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    def lengths(n, hi, lo):
        return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda").to(torch.int32)

    c, s = case, {"case": case}
    if c["op"] == "norm":
        s["x"] = normal(c["rows"], c["cols"])
        s["residual"] = normal(c["rows"], c["cols"]) if c["residual"] else None
        s["weight"] = (1 + 0.1 * torch.randn(c["cols"], generator=g, device="cuda")).to(dt)
    elif c["op"] == "cross":
        s["q"] = normal(c["batch"], c["n_q"], c["heads_q"], c["dim"])
        s["k"] = normal(c["batch"], c["n_kv"], c["heads_kv"], c["dim"])
        s["v"] = normal(c["batch"], c["n_kv"], c["heads_kv"], c["dim"])
        s["kv_len"] = lengths(c["batch"], c["n_kv"], (c["n_kv"] + 1) // 2) if c["lengths"] == "ragged" else None
        s["kv_mask"] = _mask(g, c["batch"], c["n_kv"]) if c["lengths"] == "padded" else None
        s["out"] = torch.empty_like(s["q"])
    else:
        n = c["prefixes"] * c["requests"]
        s["q"] = normal(n, c["n_q"], c["heads_q"], c["dim"])
        s["prefix_k"] = normal(c["prefixes"], c["n_prefix"], c["heads_kv"], c["dim"])
        s["prefix_v"] = normal(c["prefixes"], c["n_prefix"], c["heads_kv"], c["dim"])
        s["own_k"] = normal(n, c["n_own"], c["heads_kv"], c["dim"])
        s["own_v"] = normal(n, c["n_own"], c["heads_kv"], c["dim"])
        s["own_len"] = lengths(n, c["n_own"], c["n_q"])  # the cache's room is n_own; the last n_q keys are the queries'
        s["out"] = torch.empty_like(s["q"])
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The plan (it holds the workspace) and the output buffers that a program keeps."""
    import paper_2107_06960_gb300 as mf

    c = s["case"]
    dtype = mf.BF16 if c["dtype"] == "bf16" else mf.FP32
    if c["op"] == "norm":
        s["h"] = torch.empty_like(s["x"]) if c["residual"] else None
        s["y"] = torch.empty(s["x"].shape, device="cuda", dtype=s["x"].dtype if c["quant"] == "none" else torch.float8_e4m3fn)
        n = {"none": 0, "row": 1, "128": -(-c["cols"] // 128)}[c["quant"]]
        s["scales"] = torch.empty((c["rows"], n), device="cuda", dtype=torch.float32) if n else None
    elif c["op"] == "cross":
        s["plan"] = mf.CrossAttention(c["batch"], c["n_q"], c["n_kv"], c["heads_q"], c["heads_kv"], c["dim"], dtype=dtype)
    else:
        s["plan"] = mf.PrefixAttention(c["prefixes"], c["requests"], c["n_q"], c["n_prefix"], c["n_own"], c["heads_q"],
                                       c["heads_kv"], c["dim"], dtype=dtype)


# ---- one pass -------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "norm":
        return _plain_norm(s, c)
    if c["op"] == "cross":
        return {"out": _plain_cross(s, c)}
    return {"out": _plain_prefix(s, c)}


def _run_own(s, c):
    import paper_2107_06960_gb300 as mf

    if c["op"] == "norm":
        mf.rms_norm(s["x"], s["weight"], s["y"], residual=s["residual"], residual_out=s["h"], scales=s["scales"],
                    scale_group=128 if c["quant"] == "128" else 0, eps=EPS)
        return {k: s[k] for k in ("h", "y", "scales") if s[k] is not None}
    if c["op"] == "cross":
        s["plan"].run(s["q"], s["k"], s["v"], s["out"], kv_len=s["kv_len"], kv_mask=s["kv_mask"])
    else:
        s["plan"].run(s["q"], s["prefix_k"], s["prefix_v"], s["own_k"], s["own_v"], s["out"], own_len=s["own_len"])
    return {"out": s["out"]}


def _plain_norm(s, c):
    dt = s["x"].dtype
    h = s["x"].float()
    got = {}
    if c["residual"]:
        h = h + s["residual"].float()
        got["h"] = h.to(dt)
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    if c["quant"] == "none":
        got["y"] = y.to(dt)
        return got
    rows, cols = y.shape
    width = cols if c["quant"] == "row" else 128
    n = -(-cols // width)
    y = torch.nn.functional.pad(y, (0, n * width - cols)).view(rows, n, width)
    scales = y.abs().amax(-1) / E4M3_MAX
    scales = torch.where(scales == 0, torch.ones_like(scales), scales)
    y = (y / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).view(rows, n * width)[:, :cols]
    got["y"] = y.to(torch.float8_e4m3fn)
    got["scales"] = scales
    return got


def _plain_softmax(scores):
    """exp(scores - their maximum) and its sum, with nothing for a row that has no finite score."""
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    return p, p.sum(-1, keepdim=True)


def _plain_cross(s, c):
    B, T, S, H, Hk, D = c["batch"], c["n_q"], c["n_kv"], c["heads_q"], c["heads_kv"], c["dim"]
    q = s["q"].float().view(B, T, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, H // Hk * T, D)
    k = s["k"].float().permute(0, 2, 3, 1)
    v = s["v"].float().permute(0, 2, 1, 3)
    scores = torch.matmul(q, k) * (1 / math.sqrt(D))
    if s["kv_len"] is not None:
        scores = scores.masked_fill((torch.arange(S, device="cuda")[None] >= s["kv_len"][:, None])[:, None, None], -math.inf)
    if s["kv_mask"] is not None:
        scores = scores.masked_fill(~s["kv_mask"][:, None, None], -math.inf)
    p, total = _plain_softmax(scores)
    o = torch.where(total > 0, torch.matmul(p, v) / total, torch.zeros_like(total))
    return o.view(B, Hk, H // Hk, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H, D).to(s["q"].dtype)


def _plain_prefix(s, c):
    G, R, T, P, S = c["prefixes"], c["requests"], c["n_q"], c["n_prefix"], c["n_own"]
    H, Hk, D = c["heads_q"], c["heads_kv"], c["dim"]
    m = H // Hk
    q = s["q"].float().view(G * R, T, Hk, m, D).permute(0, 2, 3, 1, 4)  # [G*R][Hk][m][T][D]
    pk, pv = s["prefix_k"].float().permute(0, 2, 3, 1), s["prefix_v"].float().permute(0, 2, 1, 3)
    ok, ov = s["own_k"].float().permute(0, 2, 3, 1), s["own_v"].float().permute(0, 2, 1, 3)
    # the prefix once for all requests of its group, then each request's own keys
    shared = q.reshape(G, R, Hk, m * T, D).transpose(1, 2).reshape(G, Hk, R * m * T, D)
    a = torch.matmul(shared, pk).view(G, Hk, R, m * T, P).transpose(1, 2).reshape(G * R, Hk, m * T, P)
    b = torch.matmul(q.reshape(G * R, Hk, m * T, D), ok)
    last = s["own_len"][:, None] - T + torch.arange(T, device="cuda")[None]  # the last own key that query t sees
    hidden = torch.arange(S, device="cuda")[None, None] > last[:, :, None]
    b = b.view(G * R, Hk, m, T, S).masked_fill(hidden[:, None, None], -math.inf).view(G * R, Hk, m * T, S)
    p, total = _plain_softmax(torch.cat([a, b], -1) * (1 / math.sqrt(D)))
    pa, pb = p[..., :P], p[..., P:]
    pa = pa.view(G, R, Hk, m * T, P).transpose(1, 2).reshape(G, Hk, R * m * T, P)
    o = torch.matmul(pa, pv).view(G, Hk, R, m * T, D).transpose(1, 2).reshape(G * R, Hk, m * T, D)
    o = o + torch.matmul(pb, ov)
    o = torch.where(total > 0, o / total, torch.zeros_like(total))
    return o.view(G * R, Hk, m, T, D).permute(0, 3, 1, 2, 4).reshape(G * R, T, H, D).to(s["q"].dtype)


# ---- what a pass cannot do without ------------------------------------------------------------


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "norm":
        n = c["rows"] * c["cols"]
        out = e if c["quant"] == "none" else 1
        scales = {"none": 0, "row": 1, "128": -(-c["cols"] // 128)}[c["quant"]] * c["rows"] * 4
        return {"bytes": n * (e * (3 if c["residual"] else 1) + out) + c["cols"] * e + scales, "flops": 6 * n}
    H, Hk, D, T = c["heads_q"], c["heads_kv"], c["dim"], c["n_q"]
    if c["op"] == "cross":
        # half to all of a ragged or padded side is readable
        share = {"full": 1.0, "ragged": 0.75, "padded": 0.5625}[c["lengths"]]
        keys = share * c["n_kv"] * c["batch"]
        return {"bytes": 2 * c["batch"] * T * H * D * e + 2 * keys * Hk * D * e, "flops": 4 * keys * T * H * D}
    n = c["prefixes"] * c["requests"]
    mine = n * (c["n_own"] + T) / 2  # own lengths are uniform from n_q to n_own
    return {"bytes": 2 * n * T * H * D * e + 2 * (c["prefixes"] * c["n_prefix"] + mine) * Hk * D * e,
            "flops": 4 * T * H * D * (n * c["n_prefix"] + mine - n * (T - 1) / 2)}


# ---- 64 bits ------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions in double precision, one sequence and one head after another."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    if c["op"] == "norm":
        got = {}
        h = s["x"].double()
        if c["residual"]:
            h = h + s["residual"].double()
            got["h"] = h
        y = h / torch.sqrt((h * h).sum(-1, keepdim=True) / c["cols"] + EPS) * s["weight"].double()
        if c["quant"] == "none":
            return {**got, "y": y}
        width = c["cols"] if c["quant"] == "row" else 128
        blocks = y.split(width, dim=-1)
        scales = torch.cat([b.abs().amax(-1, keepdim=True) / E4M3_MAX for b in blocks], -1)
        scales[scales == 0] = 1.0
        return {**got, "y": torch.cat([b / scales[:, i : i + 1] for i, b in enumerate(blocks)], -1), "scales": scales}
    rows = s["q"].shape[0]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group = c["heads_q"] // c["heads_kv"]
    for b in range(rows):
        for h in range(c["heads_kv"]):
            q = s["q"][b, :, h * group : (h + 1) * group].double()  # [T][group][D]
            if c["op"] == "cross":
                k, v = s["k"][b, :, h].double(), s["v"][b, :, h].double()
                seen = torch.ones(c["n_kv"], dtype=torch.bool, device="cuda")
                if s["kv_len"] is not None:
                    seen &= torch.arange(c["n_kv"], device="cuda") < s["kv_len"][b]
                if s["kv_mask"] is not None:
                    seen &= s["kv_mask"][b]
                seen = seen[None].expand(c["n_q"], -1)
            else:
                f = b // c["requests"]
                k = torch.cat([s["prefix_k"][f, :, h], s["own_k"][b, :, h]]).double()
                v = torch.cat([s["prefix_v"][f, :, h], s["own_v"][b, :, h]]).double()
                at = torch.arange(c["n_prefix"] + c["n_own"], device="cuda")
                t = torch.arange(c["n_q"], device="cuda")
                seen = at[None] <= (c["n_prefix"] + s["own_len"][b] - c["n_q"] + t)[:, None]
            z = torch.einsum("tgd,sd->tgs", q, k) / math.sqrt(c["dim"])
            z = torch.where(seen[:, None], z, torch.full_like(z, -math.inf))
            z = torch.softmax(z, -1)
            z = torch.where(seen.any(-1)[:, None, None], z, torch.zeros_like(z))
            out[b, :, h * group : (h + 1) * group] = torch.einsum("tgs,sd->tgd", z, v)
    return {"out": out}
