"""Cases that stand for what a program has the operators of a drafting decoder do: a decoder that answers
over frames and verifies a tree of drafted tokens in each step, next to ``perf/operators.py``, whose
single tokens and prompts it shares the prefix attention with.

Four operators are one step of it:

``norm``    the norms around a block, with its gate and the residual's scale:
            n = x / sqrt(mean(x^2) + eps) * w1;  h = a r + b g n;  y = h / sqrt(mean(h^2) + eps) * w2,
            y in the inputs' type or in 8 bits (e4m3) with scales, one for a row or one for each 128 channels
``rotary``  positions as rotations of pairs of channels of queries and keys; keys and values go to their
            places in the request's cache
``tree``    attention of each request's drafted tokens, a tree, to its prefix (a frame's states, shared by
            neighbours), to its own earlier keys and to the tokens on the way from the tree's root
``logits``  what a request asks of its next token: penalties for repeated tokens, biases, a grammar's mask; for
            each node of the tree, whose history is the request's and the node's way from the root

Inputs are normal; projections of normalised states have unit variance.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
E4M3_MAX = 448.0
FACTOR, FIRST_POSITIONS, FAST, SLOW = 8.0, 8192, 32.0, 1.0  # of positions scaled for long contexts


def _norm(name, rows, cols, dtype, quant, post=True, gates=1):
    # quant: "none", "row" (one scale a row) or "128"; post: with the norm after the block; gates: 0 (none),
    # 1 (one for each channel) or a divisor of rows (each for rows / gates neighbours)
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "quant": quant, "post": post, "gates": gates}


def _rotary(name, batch, n_q, room, heads_q, heads_kv, dim, rot, interleaved, scaling, dtype):
    # scaling: "none", "linear" (positions divided), "base" (a larger base) or "blend" (by wavelength)
    return {"name": name, "op": "rotary", "batch": batch, "n_q": n_q, "room": room, "heads_q": heads_q, "heads_kv": heads_kv,
            "dim": dim, "rot": rot, "interleaved": interleaved, "scaling": scaling, "dtype": dtype}


def _tree(name, prefixes, requests, n_q, n_prefix, n_own, heads_q, heads_kv, dim, dtype, ragged=False):
    # ragged: requests have trees of 1 to n_q nodes
    return {"name": name, "op": "tree", "prefixes": prefixes, "requests": requests, "n_q": n_q, "n_prefix": n_prefix,
            "n_own": n_own, "heads_q": heads_q, "heads_kv": heads_kv, "dim": dim, "dtype": dtype, "ragged": ragged}


def _logits(name, batch, n_q, vocab, room, n_bias, masks, dtype, out):
    # room: of a request's history; masks: grammar states, 0: none has one
    return {"name": name, "op": "logits", "batch": batch, "n_q": n_q, "vocab": vocab, "room": room, "n_bias": n_bias,
            "masks": masks, "dtype": dtype, "out": out}


def listed():
    return [
        # one decoding step of 16 requests: latency
        _norm("norm_step_16x1024", 16, 1024, "bf16", "row"),
        # the states of eight frames at 1216 pixels in 1024 channels, a gate for each frame
        _norm("norm_b8_1216_1024", 8 * 5776, 1024, "bf16", "none", gates=8),
        # odd sizes in single precision, without a norm behind the block
        _norm("norm_fp32_1443x1001", 1443, 1001, "fp32", "none", post=False),
        # one token of each of 64 requests: latency
        _rotary("rotary_step_b64", 64, 1, 600, 32, 8, 128, 128, False, "none", "bf16"),
        # long prompts at far positions, scaled by wavelength
        _rotary("rotary_prompt_8x2048", 8, 2048, 2100, 32, 8, 128, 128, False, "blend", "bf16"),
        # odd lengths, part of each head, neighbouring channels as pairs, single precision
        _rotary("rotary_fp32_3x333", 3, 333, 401, 8, 2, 80, 40, True, "linear", "fp32"),
        # the smallest: one request drafts eight tokens about one 608x608 frame
        _tree("tree_608_r1x8", 1, 1, 8, 1444, 96, 16, 4, 64, "bf16"),
        # a server's step: 64 requests draft 16 tokens each about a clip of sixteen 608x608 frames
        _tree("tree_clip_r64x16", 1, 64, 16, 16 * 1444, 512, 32, 8, 128, "bf16"),
        # trees of unequal sizes up to 61, eight requests about each of four frames at 1216 pixels
        _tree("tree_1216_4x8x61", 4, 8, 61, 5776, 200, 16, 4, 128, "bf16", ragged=True),
        # a step of 16 requests before the choice of a token: latency
        _logits("logits_step_16x32000", 16, 1, 32000, 512, 16, 0, "bf16", "fp32"),
        # the largest: trees of 16 nodes of 64 requests, half of them under a grammar
        _logits("logits_r64x16_131072", 64, 16, 131072, 2048, 64, 256, "bf16", "bf16"),
        # rows of an odd number of logits, long histories, single precision
        _logits("logits_fp32_7x50001", 7, 1, 50001, 20000, 300, 7, "fp32", "fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "rotary", "rotary", "tree", "tree", "tree", "logits", "logits"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "norm":
        cols = rng.choice([_log_int(rng, 64, 4096), 8 * _log_int(rng, 8, 1024)])
        rows = min(_log_int(rng, 1, 50000), max(1, (46_000_000 if dtype == "bf16" else 23_000_000) // cols))
        per = rng.choice([0, 1, rows, rng.randint(1, rows)])  # rows that share a gate
        gates = 0 if per == 0 else max(1, rows // per)
        c = _norm("", gates * (rows // gates) if gates else rows, cols, dtype, rng.choice(["none", "none", "row", "128"]),
                  rng.random() < 0.7, gates)
    elif op == "rotary":
        dim = rng.choice([64, 64, 128, 128, 80, 40])
        heads_kv = rng.choice([1, 2, 4, 8])
        heads_q = heads_kv * rng.choice([1, 2, 4, 8])
        most = (90_000_000 if dtype == "bf16" else 45_000_000) // ((heads_q + 4 * heads_kv) * dim)
        n_q = 1 if rng.random() < 0.3 else min(_log_int(rng, 2, 4096), most)
        batch = max(1, min(_log_int(rng, 1, 128), most // n_q))
        room = n_q + rng.randint(0, min(2000, max(1, 2 * most // batch - n_q)))
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        c = _rotary("", batch, n_q, room, heads_q, heads_kv, dim, rot, rng.random() < 0.4,
                    rng.choice(["none", "none", "linear", "base", "blend"]) if rot > 2 else "none", dtype)
    elif op == "tree":
        dim = rng.choice([64, 64, 128, 128, 80, 40])
        heads_kv = rng.choice([1, 2, 4, 8])
        heads_q = heads_kv * rng.choice([1, 2, 4, 8])
        pairs = (60_000_000 if dtype == "fp32" else 700_000_000) // heads_q
        keys = (24_000_000 if dtype == "fp32" else 40_000_000) // (heads_kv * dim)
        n_prefix = min(_log_int(rng, 16, 24000), keys // 2)
        n_q = _log_int(rng, 1, 100)
        n_own = n_q + _log_int(rng, 1, 600)
        both = n_prefix + n_own
        prefixes = max(1, min(_log_int(rng, 1, 8), keys // (2 * n_prefix), pairs // (n_q * both)))
        requests = max(1, min(_log_int(rng, 1, 64), keys // (2 * n_own * prefixes), pairs // (n_q * both * prefixes)))
        c = _tree("", prefixes, requests, n_q, n_prefix, n_own, heads_q, heads_kv, dim, dtype, rng.random() < 0.5)
    else:
        vocab = rng.choice([_log_int(rng, 500, 200000), 64 * _log_int(rng, 16, 3000)])
        out = rng.choice([dtype, "fp32"])
        most = 520_000_000 // ((2 if dtype == "bf16" else 4) + (2 if out == "bf16" else 4)) // vocab
        n_q = min(rng.choice([1, 1, _log_int(rng, 2, 64)]), most)
        batch = max(1, min(_log_int(rng, 1, 128), most // n_q))
        room = _log_int(rng, 1, 30000)
        c = _logits("", batch, n_q, vocab, room, rng.choice([0, 0, _log_int(rng, 1, 300)]),
                    rng.choice([0, 1, _log_int(rng, 2, 300)]), dtype, out)
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------


def _trees(g, n, n_q):
    """Random trees of n_q nodes: a node's parent is an earlier one or, for a tenth of them, the text before
    the tree.  [n][n_q][n_q]: whether node j is on the way from the root to node t, t itself among them."""
    parent = (torch.rand(n, n_q, generator=g, device="cuda") * torch.arange(n_q, device="cuda")).long()
    free = torch.rand(n, n_q, generator=g, device="cuda") < 0.1
    way = torch.zeros(n, n_q, n_q, dtype=torch.bool, device="cuda")
    at = torch.arange(n, device="cuda")
    for t in range(n_q):
        if t > 0:
            way[:, t] = way[at, parent[:, t]] & ~free[:, t, None]
        way[:, t, t] = True
    return way


def _bits(flags):
    """[...][n] truth values as [...][ceil(n / 32)] words, the first in the lowest bit."""
    n = flags.shape[-1]
    words = -(-n // 32)
    x = torch.nn.functional.pad(flags.long(), (0, words * 32 - n)).view(flags.shape[:-1] + (words, 32))
    x = (x << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    def ints(lo, hi, *shape):  # hi is one of them
        return torch.randint(lo, hi + 1, shape, generator=g, device="cuda").to(torch.int32)

    c, s = case, {"case": case}
    if c["op"] == "norm":
        s["x"], s["residual"] = normal(c["rows"], c["cols"]), normal(c["rows"], c["cols"])
        near_one = [(1 + 0.1 * torch.randn(c["cols"], generator=g, device="cuda")).to(dt) for _ in range(2)]
        s["post_weight"], s["weight"] = near_one[0] if c["post"] else None, near_one[1]
        s["gate"] = normal(c["gates"], c["cols"]) if c["gates"] else None
        s["h"] = torch.empty_like(s["x"])
        s["y"] = torch.empty(s["x"].shape, device="cuda", dtype=dt if c["quant"] == "none" else torch.float8_e4m3fn)
        n = {"none": 0, "row": 1, "128": -(-c["cols"] // 128)}[c["quant"]]
        s["scales"] = torch.empty((c["rows"], n), device="cuda", dtype=torch.float32) if n else None
    elif c["op"] == "rotary":
        B, T, H, Hk, D = c["batch"], c["n_q"], c["heads_q"], c["heads_kv"], c["dim"]
        # queries, keys and values side by side, as one product leaves them
        qkv = normal(B, T, H + 2 * Hk, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:]
        s["q_out"] = torch.empty(B, T, H, D, device="cuda", dtype=dt)
        s["k_cache"], s["v_cache"] = normal(B, c["room"], Hk, D), normal(B, c["room"], Hk, D)
        first = ints(0, c["room"] - T, B)
        s["places"] = first[:, None] + torch.arange(T, device="cuda", dtype=torch.int32)
        # a long text, or a clip, stands before a request's cache
        s["positions"] = s["places"] + ints(0, 100000, B)[:, None]
    elif c["op"] == "tree":
        n, T = c["prefixes"] * c["requests"], c["n_q"]
        H, Hk, D = c["heads_q"], c["heads_kv"], c["dim"]
        s["q"] = normal(n, T, H, D)
        s["prefix_k"], s["prefix_v"] = normal(c["prefixes"], c["n_prefix"], Hk, D), normal(c["prefixes"], c["n_prefix"], Hk, D)
        s["own_k"], s["own_v"] = normal(n, c["n_own"], Hk, D), normal(n, c["n_own"], Hk, D)
        s["nodes"] = ints(1, T, n) if c["ragged"] else None
        # the tree's keys stand behind the request's earlier ones, of which the cache holds any number
        before = (torch.rand(n, generator=g, device="cuda") * (c["n_own"] - T + 1)).to(torch.int32)
        s["own_len"] = before + (s["nodes"] if c["ragged"] else T)
        s["tree"] = _bits(_trees(g, n, T))
        s["out"] = torch.empty_like(s["q"])
    else:
        B, T, V = c["batch"], c["n_q"], c["vocab"]
        s["logits"] = (3 * torch.randn((B, T, V), generator=g, device="cuda")).to(dt)
        s["out"] = torch.empty((B, T, V), device="cuda", dtype=_DT[c["out"]])
        # texts repeat themselves: common tokens are drawn more often
        s["tokens"] = (V * torch.rand((B, c["room"]), generator=g, device="cuda").pow(3)).to(torch.int32).clamp(max=V - 1)
        s["lengths"] = ints(c["room"] // 2, c["room"], B)
        s["prompt_lengths"] = (s["lengths"] * torch.rand(B, generator=g, device="cuda")).to(torch.int32)
        s["repetition"] = 1 + 0.3 * torch.rand(B, generator=g, device="cuda")
        s["presence"], s["frequency"] = [torch.rand(B, generator=g, device="cuda") - 0.2 for _ in range(2)]
        s["drafts"] = s["tree"] = s["bias_ids"] = s["bias"] = s["masks"] = s["mask_rows"] = None
        if T > 1:
            s["drafts"] = (V * torch.rand((B, T), generator=g, device="cuda").pow(3)).to(torch.int32).clamp(max=V - 1)
            s["tree"] = _bits(_trees(g, B, T))
        if c["n_bias"]:
            # an id once: random steps of at least one, unused places -1
            steps = torch.randint(1, max(2, V // c["n_bias"]) + 1, (B, c["n_bias"]), generator=g, device="cuda")
            ids = steps.cumsum(-1)
            s["bias_ids"] = torch.where(ids < V, ids, torch.full_like(ids, -1)).to(torch.int32)
            s["bias"] = 2 * torch.randn((B, c["n_bias"]), generator=g, device="cuda")
        if c["masks"]:
            # a grammar allows few tokens or most
            share = torch.rand((c["masks"], 1), generator=g, device="cuda")
            s["masks"] = torch.cat([_bits(torch.rand((1, V), generator=g, device="cuda") < x) for x in share])
            rows = ints(0, c["masks"] - 1, B, T)
            s["mask_rows"] = torch.where(ints(0, 1, B, 1) > 0, rows, torch.full_like(rows, -1))
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The plan that a program keeps: the table of frequencies, or the workspace."""
    import paper_2107_06960_gb300 as mf

    c = s["case"]
    dtype = mf.BF16 if c["dtype"] == "bf16" else mf.FP32
    if c["op"] == "rotary":
        scaling = {"none": mf.ROTARY_PLAIN, "linear": mf.ROTARY_LINEAR, "base": mf.ROTARY_BASE, "blend": mf.ROTARY_BLEND}[c["scaling"]]
        s["plan"] = mf.Rotary(c["dim"], c["rot"], dtype=dtype, interleaved=c["interleaved"], scaling=scaling,
                              factor=1.0 if c["scaling"] == "none" else FACTOR,
                              first_positions=FIRST_POSITIONS if c["scaling"] == "blend" else 0, fast=FAST, slow=SLOW)
    elif c["op"] == "tree":
        s["plan"] = mf.TreeAttention(c["prefixes"], c["requests"], c["n_q"], c["n_prefix"], c["n_own"], c["heads_q"],
                                     c["heads_kv"], c["dim"], dtype=dtype)


# ---- one pass -------------------------------------------------------------------------------

BRANCH, RESIDUAL = 0.7, 0.9  # scales of a block's result and of the residual


def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "tree": _plain_tree, "logits": _plain_logits}[c["op"]](s, c)


def _run_own(s, c):
    import paper_2107_06960_gb300 as mf

    if c["op"] == "norm":
        mf.block_norm(s["x"], s["residual"], s["h"], post_weight=s["post_weight"], gate=s["gate"], branch_scale=BRANCH,
                      residual_scale=RESIDUAL, weight=s["weight"], y=s["y"], scales=s["scales"],
                      scale_group=128 if c["quant"] == "128" else 0, eps=EPS)
        return {k: s[k] for k in ("h", "y", "scales") if s[k] is not None}
    if c["op"] == "rotary":
        s["plan"].run(s["positions"], q=s["q"], q_out=s["q_out"], k=s["k"], k_out=s["k_cache"], v=s["v"],
                      v_out=s["v_cache"], places=s["places"])
        return {k: s[k] for k in ("q_out", "k_cache", "v_cache")}
    if c["op"] == "tree":
        s["plan"].run(s["q"], s["prefix_k"], s["prefix_v"], s["own_k"], s["own_v"], s["tree"], s["out"], nodes=s["nodes"],
                      own_len=s["own_len"])
    else:
        mf.adjust_logits(s["logits"], s["out"], tokens=s["tokens"], lengths=s["lengths"], prompt_lengths=s["prompt_lengths"],
                         repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], drafts=s["drafts"],
                         tree=s["tree"], bias_ids=s["bias_ids"], bias=s["bias"], masks=s["masks"], mask_rows=s["mask_rows"])
    return {"out": s["out"]}


def _plain_norm(s, c):
    dt = s["x"].dtype
    n = s["x"].float()
    if c["post"]:
        n = n * torch.rsqrt(n.square().mean(-1, keepdim=True) + EPS) * s["post_weight"].float()
    if c["gates"]:
        n = (n.view(c["gates"], -1, c["cols"]) * s["gate"].float()[:, None]).view(n.shape)
    h = RESIDUAL * s["residual"].float() + BRANCH * n
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    got = {"h": h.to(dt)}
    if c["quant"] == "none":
        return {**got, "y": y.to(dt)}
    rows, cols = y.shape
    width = cols if c["quant"] == "row" else 128
    n = -(-cols // width)
    y = torch.nn.functional.pad(y, (0, n * width - cols)).view(rows, n, width)
    scales = y.abs().amax(-1) / E4M3_MAX
    scales = torch.where(scales == 0, torch.ones_like(scales), scales)
    y = (y / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).view(rows, n * width)[:, :cols]
    return {**got, "y": y.to(torch.float8_e4m3fn), "scales": scales}


def _frequencies(c):
    """Radians a position of each pair, and the rotated channels' factor."""
    rot, base = c["rot"], 10000.0
    if c["scaling"] == "base":
        base *= FACTOR ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    if c["scaling"] == "linear":
        f = f / FACTOR
    if c["scaling"] == "blend":  # pairs that turn often within the first positions keep their frequency
        keep = ((FIRST_POSITIONS * f / (2 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0, 1)
        f = f * (keep + (1 - keep) / FACTOR)
    return f, 0.1 * math.log(FACTOR) + 1 if c["scaling"] == "blend" else 1.0


def _plain_rotary(s, c):
    f, m = _frequencies(c)
    angle = s["positions"].double()[..., None] * f  # far positions lose their angle in 32 bits
    cos, sin = (m * torch.cos(angle)).float()[:, :, None], (m * torch.sin(angle)).float()[:, :, None]
    rot = c["rot"]

    def turn(x):
        x = x.float()
        if c["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([y, x[..., rot:]], -1)

    at = torch.arange(c["batch"], device="cuda")[:, None], s["places"].long()
    s["q_out"].copy_(turn(s["q"]))
    s["k_cache"][at] = turn(s["k"]).to(s["k"].dtype)
    s["v_cache"][at] = s["v"]
    return {k: s[k] for k in ("q_out", "k_cache", "v_cache")}


def _flags(words, n):
    """_bits() back."""
    return ((words.long()[..., None] >> torch.arange(32, device="cuda")) & 1).bool().flatten(-2)[..., :n]


def _plain_tree(s, c):
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
    nodes = torch.full_like(s["own_len"], T) if s["nodes"] is None else s["nodes"]
    node = torch.arange(S, device="cuda")[None] - (s["own_len"] - nodes)[:, None].long()  # of each own key; negative: before the tree
    way = torch.gather(_flags(s["tree"], T), 2, node.clamp(0, T - 1)[:, None].expand(-1, T, -1))
    seen = (node < 0)[:, None] | (way & (node < nodes[:, None])[:, None])
    b = b.view(G * R, Hk, m, T, S).masked_fill(~seen[:, None, None], -math.inf).view(G * R, Hk, m * T, S)
    z = torch.cat([a, b], -1) * (1 / math.sqrt(D))
    p = torch.exp(z - z.amax(-1, keepdim=True))
    total = p.sum(-1, keepdim=True)
    pa, pb = p[..., :P], p[..., P:]
    pa = pa.view(G, R, Hk, m * T, P).transpose(1, 2).reshape(G, Hk, R * m * T, P)
    o = torch.matmul(pa, pv).view(G, Hk, R, m * T, D).transpose(1, 2).reshape(G * R, Hk, m * T, D)
    o = (o + torch.matmul(pb, ov)) / total
    o = o.view(G * R, Hk, m, T, D).permute(0, 3, 1, 2, 4).reshape(G * R, T, H, D)
    live = torch.arange(T, device="cuda")[None] < nodes[:, None]  # rows past a tree's nodes are zero
    return {"out": torch.where(live[:, :, None, None], o, torch.zeros_like(o)).to(s["q"].dtype)}


def _plain_logits(s, c):
    B, T, V = c["batch"], c["n_q"], c["vocab"]
    at = torch.arange(c["room"], device="cuda")[None]
    here, prompt = at < s["lengths"][:, None], at < s["prompt_lengths"][:, None]
    ids = s["tokens"].long()
    before = torch.zeros(B, V, device="cuda").scatter_add_(1, ids, (here & prompt).float())[:, None]
    count = torch.zeros(B, V, device="cuda").scatter_add_(1, ids, (here & ~prompt).float())[:, None].repeat(1, T, 1)
    if s["drafts"] is not None:
        count.scatter_add_(2, s["drafts"].long()[:, None].expand(B, T, T), _flags(s["tree"], T).float())
    x = s["logits"].float()
    r = s["repetition"][:, None, None]
    x = torch.where((count > 0) | (before > 0), torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None, None] * count - s["presence"][:, None, None] * (count > 0)
    if s["bias"] is not None:
        held = s["bias_ids"] >= 0
        x = x + torch.zeros(B, V, device="cuda").scatter_add_(1, s["bias_ids"].clamp(min=0).long(), s["bias"] * held)[:, None]
    if s["masks"] is not None:
        allowed = _flags(s["masks"], V)[s["mask_rows"].clamp(min=0).long()] | (s["mask_rows"] < 0)[..., None]
        x = x.masked_fill(~allowed, -math.inf)
    s["out"].copy_(x)
    return {"out": s["out"]}


# ---- what a pass cannot do without ------------------------------------------------------------


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "norm":
        n = c["rows"] * c["cols"]
        out = e if c["quant"] == "none" else 1
        scales = {"none": 0, "row": 1, "128": -(-c["cols"] // 128)}[c["quant"]] * c["rows"] * 4
        return {"bytes": n * (3 * e + out) + (1 + c["post"] + c["gates"]) * c["cols"] * e + scales, "flops": 14 * n}
    if c["op"] == "rotary":
        tokens = c["batch"] * c["n_q"]
        heads = c["heads_q"] + c["heads_kv"]
        return {"bytes": 2 * tokens * (heads + c["heads_kv"]) * c["dim"] * e + 8 * tokens, "flops": 3 * tokens * heads * c["rot"]}
    if c["op"] == "tree":
        H, Hk, D, T = c["heads_q"], c["heads_kv"], c["dim"], c["n_q"]
        n = c["prefixes"] * c["requests"]
        nodes = (T + 1) / 2 if c["ragged"] else T
        before = (c["n_own"] - T) / 2
        rows = n * nodes * H
        # a tree's node has about as many on its way as its logarithm says
        return {"bytes": n * T * H * D * e + rows * D * e + 2 * (c["prefixes"] * c["n_prefix"] + n * (before + nodes)) * Hk * D * e,
                "flops": 4 * D * rows * (c["n_prefix"] + before + math.log2(nodes + 1))}
    n = c["batch"] * c["n_q"] * c["vocab"]
    o = 2 if c["out"] == "bf16" else 4
    states = min(c["masks"], c["batch"] * c["n_q"])
    return {"bytes": n * (e + o) + c["batch"] * (3 * c["room"] + 8 * c["n_bias"]) + states * c["vocab"] // 8, "flops": 2 * n}


# ---- 64 bits ------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions in double precision, one request after another."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "rotary": _exact_rotary, "tree": _exact_tree, "logits": _exact_logits}[case["op"]](s, case)


def _exact_norm(s, c):
    def normed(x, w):
        return x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["cols"] + EPS) * w.double()

    n = s["x"].double()
    if c["post"]:
        n = normed(n, s["post_weight"])
    if c["gates"]:
        n = n * s["gate"].double().repeat_interleave(c["rows"] // c["gates"], 0)
    h = RESIDUAL * s["residual"].double() + BRANCH * n
    y = normed(h, s["weight"])
    if c["quant"] == "none":
        return {"h": h, "y": y}
    blocks = y.split(c["cols"] if c["quant"] == "row" else 128, dim=-1)
    scales = torch.cat([b.abs().amax(-1, keepdim=True) / E4M3_MAX for b in blocks], -1)
    scales[scales == 0] = 1.0
    return {"h": h, "y": torch.cat([b / scales[:, i : i + 1] for i, b in enumerate(blocks)], -1), "scales": scales}


def _exact_rotary(s, c):
    rot, got = c["rot"], {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
    pairs = []
    for i in range(rot // 2):
        base = 10000.0 * (FACTOR ** (rot / (rot - 2)) if c["scaling"] == "base" else 1.0)
        f = base ** (-2 * i / rot)
        if c["scaling"] == "linear":
            f /= FACTOR
        if c["scaling"] == "blend":
            share = min(1.0, max(0.0, (FIRST_POSITIONS * f / (2 * math.pi) - SLOW) / (FAST - SLOW)))
            f = share * f + (1 - share) * f / FACTOR
        pairs.append(((2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2), f))
    m = 1 + 0.1 * math.log(FACTOR) if c["scaling"] == "blend" else 1.0

    def turned(x):
        x = x.double()
        y = x.clone()
        for (i, j), f in pairs:
            w = torch.polar(torch.full_like(s["positions"], m, dtype=torch.float64), s["positions"].double() * f)
            z = torch.complex(x[..., i], x[..., j]) * w[:, :, None]
            y[..., i], y[..., j] = z.real, z.imag
        return y

    got["q_out"] = turned(s["q"])
    k = turned(s["k"])
    for b in range(c["batch"]):
        got["k_cache"][b].index_copy_(0, s["places"][b].long(), k[b])
        got["v_cache"][b].index_copy_(0, s["places"][b].long(), s["v"][b].double())
    return {k: got[k] for k in ("q_out", "k_cache", "v_cache")}


def _exact_tree(s, c):
    T, group = c["n_q"], c["heads_q"] // c["heads_kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    words = s["tree"].cpu().tolist()
    lengths = s["own_len"].cpu().tolist()
    for b in range(c["prefixes"] * c["requests"]):
        n = T if s["nodes"] is None else int(s["nodes"][b])
        before = lengths[b] - n
        # only what each node reads: the prefix, the keys before the tree, and by their bits the tree's own
        seen = torch.zeros(n, c["n_prefix"] + before + n, dtype=torch.bool)
        seen[:, : c["n_prefix"] + before] = True
        seen[:, c["n_prefix"] + before:] = torch.tensor([[words[b][t][j // 32] >> (j % 32) & 1 for j in range(n)] for t in range(n)]) > 0
        seen = seen.cuda()
        f = b // c["requests"]
        for h in range(c["heads_kv"]):
            k = torch.cat([s["prefix_k"][f, :, h], s["own_k"][b, : lengths[b], h]]).double()
            v = torch.cat([s["prefix_v"][f, :, h], s["own_v"][b, : lengths[b], h]]).double()
            q = s["q"][b, :n, h * group : (h + 1) * group].double()
            z = torch.einsum("tgd,sd->tgs", q, k) / math.sqrt(c["dim"])
            z = torch.softmax(torch.where(seen[:, None], z, torch.full_like(z, -math.inf)), -1)
            out[b, :n, h * group : (h + 1) * group] = torch.einsum("tgs,sd->tgd", z, v)
    return {"out": out}


def _exact_logits(s, c):
    B, T, V = c["batch"], c["n_q"], c["vocab"]
    out = s["logits"].double()
    for b in range(B):
        text = s["tokens"][b, : int(s["lengths"][b])].long()
        split = min(int(s["prompt_lengths"][b]), text.numel())
        said = torch.bincount(text[:split], minlength=V)
        for t in range(T):
            ids = text[split:]
            if s["drafts"] is not None:
                words = s["tree"][b, t].cpu().tolist()
                way = [j for j in range(T) if words[j // 32] >> (j % 32) & 1]
                ids = torch.cat([ids, s["drafts"][b].long()[way]])
            n = torch.bincount(ids, minlength=V)
            x, r = out[b, t], s["repetition"][b].double()
            hit = torch.nonzero((n + said) > 0)[:, 0]
            x[hit] = torch.where(x[hit] > 0, x[hit] / r, x[hit] * r)
            x -= s["frequency"][b].double() * n + s["presence"][b].double() * (n > 0)
            if s["bias"] is not None:
                held = torch.nonzero(s["bias_ids"][b] >= 0)[:, 0]
                x.index_add_(0, s["bias_ids"][b, held].long(), s["bias"][b, held].double())
            row = -1 if s["mask_rows"] is None else int(s["mask_rows"][b, t])
            if row >= 0:
                at = torch.arange(V, device="cuda")
                x[(s["masks"][row].long()[at // 32] >> (at % 32)) & 1 == 0] = -math.inf
    return {"out": out}
