"""Penalties, biases and grammar masks against their definition in 64 bits, one row after another."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from draft_util import random_ways, words  # noqa: E402


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _reference(x, said, prompt, extra, r, p, f, bias, allowed):
    """One row (host lists and tensors): its values, and the sizes that roundings are relative to."""
    V = x.numel()
    before, n = torch.zeros(V, dtype=torch.float64), torch.zeros(V, dtype=torch.float64)
    for i, t in enumerate(said):
        if 0 <= t < V:
            (before if i < prompt else n)[t] += 1
    for t in extra:
        if 0 <= t < V:
            n[t] += 1
    x = x.double()
    y = torch.where((before + n) > 0, torch.where(x > 0, x / r, x * r), x)
    size = y.abs() + f.__abs__() * n + abs(p) * (n > 0)
    y = y - f * n - p * (n > 0)
    changed = (before + n) > 0
    last = {i: b for i, b in bias if 0 <= i < V}
    for i, b in last.items():
        y[i] += b
        size[i] += abs(b)
        changed[i] = True
    if allowed is not None:
        y = torch.where(allowed, y, torch.full_like(y, -math.inf))
    return y, size, changed


def _logits(mf, B, T, V, dt, out_dt=None, room=0, n_bias=0, n_masks=0, drafts=None, shared=(False, False), pad=(0, 0), seed=1,
            lengths=None, prompts=None, penalties="rpf", mask_rows="some", in_place=False, two_dims=False):
    g = torch.Generator()
    g.manual_seed(seed)
    logits = torch.empty((B, T, V + pad[0]), dtype=dt, device="cuda")[..., :V]
    logits.copy_(3 * torch.randn((B, T, V), generator=g))
    out = logits if in_place else torch.empty((B, T, V + pad[1]), dtype=out_dt or dt, device="cuda")[..., :V]
    was = logits.cpu().clone()

    def ids(*shape):  # some outside the vocabulary, many twice
        x = torch.randint(-2, max(2, V // 3) + 1, shape, generator=g)
        return torch.where(torch.rand(shape, generator=g) < 0.1, torch.randint(0, 2 ** 31 - 1, shape, generator=g), x).to(torch.int32)

    def floats(lo, hi):
        return lo + (hi - lo) * torch.rand(B, generator=g)
    a = {}
    tokens = ids(B, room) if room else None
    lens, firsts = lengths or [room] * B, prompts or [0] * B
    if room:
        a["tokens"] = tokens
        if lengths:
            a["lengths"] = torch.tensor(lengths, dtype=torch.int32)
        if prompts:
            a["prompt_lengths"] = torch.tensor(prompts, dtype=torch.int32)
    r, p, f = floats(0.7, 1.6), floats(-0.5, 0.9), floats(-0.3, 0.6)
    for c, name, x in (("r", "repetition", r), ("p", "presence", p), ("f", "frequency", f)):
        if c in penalties:
            a[name] = x
        else:
            x.fill_(1.0 if c == "r" else 0.0)
    way = None
    if drafts:
        a["drafts"] = ids(B, T)
        way = random_ways(1 if shared[0] else B, T, seed)
        if drafts == "tree":
            a["tree"] = words(way)
        else:
            way = torch.ones(T, T, dtype=torch.bool).tril()[None]
    if n_bias:
        n = 1 if shared[1] else B
        a["bias_ids"], a["bias"] = ids(n, n_bias), torch.randn((n, n_bias), generator=g)
    allow = rows = None
    if n_masks:
        allow = torch.rand((n_masks, V), generator=g) < torch.rand((n_masks, 1), generator=g)
        allow[0] = False
        a["masks"] = words(allow)
        if mask_rows == "some":
            rows = torch.randint(-1, n_masks + 1, (B, T), generator=g).to(torch.int32)  # n_masks: none, as -1
            a["mask_rows"] = rows
        else:
            rows = torch.arange(B * T).view(B, T)
    x, o = (logits[:, 0], out[:, 0]) if two_dims else (logits, out)
    if two_dims and rows is not None and "mask_rows" in a:
        a["mask_rows"] = a["mask_rows"][:, 0].contiguous()
    mf.adjust_logits(x, o, **{k: t.cuda() for k, t in a.items()})
    got = out.cpu()
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    for b in range(B):
        said = tokens[b, :min(max(lens[b], 0), room)].tolist() if room else []
        bias = []
        if n_bias:
            i = 0 if shared[1] else b
            bias = list(zip(a["bias_ids"][i].tolist(), a["bias"][i].double().tolist()))
        for t in range(T):
            extra = []
            if drafts:
                extra = a["drafts"][b][way[b if way.shape[0] > 1 else 0, t]].tolist()
            allowed = allow[rows[b, t]] if n_masks and 0 <= rows[b, t] < n_masks else None
            ref, size, changed = _reference(was[b, t], said, firsts[b], extra, r[b].item(), p[b].item(), f[b].item(), bias, allowed)
            y = got[b, t].double()
            assert torch.equal(y == -math.inf, ref == -math.inf)
            fine = ref != -math.inf
            # five fp32 operations, each half a step of what has been summed, then the result's rounding
            tol = 5 * 2.0 ** -24 * size + half * (ref.abs() + 2.0 ** -21 * size)
            assert ((y - ref).abs()[fine] <= tol[fine]).all(), (b, t)
            assert torch.equal(got[b, t][fine & ~changed], was[b, t].to(out.dtype)[fine & ~changed])


TYPES = [(torch.bfloat16, None), (torch.bfloat16, torch.float32), (torch.float32, None)]


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("B,T,V,room", [(1, 1, 1, 1), (2, 1, 7, 5), (1, 1, 8, 0), (3, 2, 1000, 33), (2, 1, 8192, 100), (1, 3, 8193, 64), (2, 1, 50001, 3000), (5, 1, 4096, 4000), (1, 1, 131072, 20)])
def test_sizes(mf, dt, out_dt, B, T, V, room):
    _logits(mf, B, T, V, dt, out_dt, room=room)
    _logits(mf, B, T, V, dt, out_dt, room=room, n_bias=5, n_masks=3, drafts="tree")


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("penalties", ["", "r", "p", "f", "pf", "rpf"])
def test_penalties(mf, dt, out_dt, penalties):
    """Histories of no token, one, all and more than there is room for; prompts alike."""
    _logits(mf, 6, 1, 500, dt, out_dt, room=200, lengths=[0, 1, 200, 999, -4, 120], prompts=[0, 1, 100, 300, 5, -2], penalties=penalties)


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("drafts", ["tree", "chain"])
@pytest.mark.parametrize("T", [1, 31, 33, 70])
@pytest.mark.parametrize("shared", [False, True])
def test_drafted_tokens(mf, dt, out_dt, drafts, T, shared):
    _logits(mf, 3, T, 300, dt, out_dt, room=40, lengths=[40, 0, 13], prompts=[10, 0, 13], drafts=drafts, shared=(shared, False))


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("n_bias", [1, 300, 4095])
@pytest.mark.parametrize("shared", [False, True])
def test_biases(mf, dt, out_dt, n_bias, shared):
    """Ids that are there many times: the last counts."""
    _logits(mf, 3, 2, 1500, dt, out_dt, room=50, n_bias=n_bias, shared=(False, shared))


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("V", [31, 32, 33, 1000, 50001])
@pytest.mark.parametrize("mask_rows", ["some", "each"])
def test_masks(mf, dt, out_dt, V, mask_rows):
    _logits(mf, 2, 4, V, dt, out_dt, room=10, n_masks=8, mask_rows=mask_rows)


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("pad", [(0, 1), (1, 0), (3, 5), (8, 16), (7, 7)])
@pytest.mark.parametrize("V", [1001, 4096])
def test_strides(mf, dt, out_dt, pad, V):
    _logits(mf, 2, 3, V, dt, out_dt, room=60, n_bias=3, n_masks=2, pad=pad)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1001, 20000])
@pytest.mark.parametrize("n_masks", [0, 4])
def test_in_place(mf, dt, V, n_masks):
    _logits(mf, 3, 2, V, dt, room=500, n_bias=7, n_masks=n_masks, drafts="tree", in_place=True)
    _logits(mf, 3, 1, V, dt, room=500, n_masks=n_masks, in_place=True, two_dims=True)


def test_values_at_the_ends(mf):
    """Infinities and NaN stay where they are, except where the mask forbids; nothing asked for: a copy."""
    x = torch.tensor([[math.inf, -math.inf, math.nan, 0.0, -0.0, 3e38, -3e38, 1.0]], device="cuda")
    o = torch.empty_like(x)
    mf.adjust_logits(x, o)
    assert torch.equal(o.view(torch.int32), x.view(torch.int32))
    tokens = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    mf.adjust_logits(x, o, tokens=tokens, repetition=torch.tensor([2.0], device="cuda"),
                     masks=torch.tensor([[0b01111011]], dtype=torch.int32, device="cuda"))
    assert o[0].tolist()[:2] == [math.inf, -math.inf] and o[0, 2] == -math.inf and o[0, 7] == -math.inf
    assert o[0, 3] == 0 and o[0, 4] == 0 and o[0, 5] == x[0, 5] / 2 and o[0, 6] == -math.inf
    tokens = torch.full((1, 100000), 7, dtype=torch.int32, device="cuda")  # one token many times
    mf.adjust_logits(x, o, tokens=tokens, frequency=torch.tensor([0.5], device="cuda"))
    assert o[0, 7] == 1.0 - 50000


def test_no_rows(mf):
    z = torch.empty((0, 3, 100), device="cuda")
    mf.adjust_logits(z, torch.empty_like(z))


def test_one_result_a_call(mf):
    """The order in which a history is counted does not show."""
    x = torch.randn((4, 40000), device="cuda")
    t = torch.randint(0, 50, (4, 5000), device="cuda").to(torch.int32)
    p = torch.full((4,), 0.37, device="cuda")
    outs = [torch.empty_like(x) for _ in range(5)]
    for o in outs:
        mf.adjust_logits(x, o, tokens=t, repetition=p + 1, presence=p, frequency=p)
    assert all(torch.equal(outs[0], o) for o in outs[1:])


@pytest.mark.parametrize("room,V", [(30, 5000), (3000, 20000), (9000, 20000), (9000, 900000), (17000, 1200000)])
def test_captured(mf, room, V):  # of 16 rows
    """Each form of the kernel in a graph, replayed on other histories and logits, on a stream of its own."""
    x = torch.randn((2, 8, V), device="cuda").to(torch.bfloat16)
    tokens = torch.randint(0, V, (2, room), device="cuda").to(torch.int32)
    drafts = torch.randint(0, V, (2, 8), device="cuda").to(torch.int32)
    length = torch.full((2,), room, dtype=torch.int32, device="cuda")
    p, out, want = torch.full((2,), 1.2, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            mf.adjust_logits(x, out, tokens=tokens, lengths=length, repetition=p, drafts=drafts)
        for seed in range(3):
            x.copy_(torch.randn(x.shape, device="cuda"))
            tokens.copy_(torch.randint(0, V, tokens.shape, device="cuda"))
            length.copy_(torch.randint(0, room + 1, (2,), device="cuda"))
            g.replay()
            mf.adjust_logits(x, want, tokens=tokens, lengths=length, repetition=p, drafts=drafts)
            stream.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and not torch.equal(out, x)


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("B,T,V,room", [(3, 2, 5000, 9000), (2, 5, 4100, 2049), (2, 3, 9001, 8193), (1, 17, 1000001, 17000)])
def test_long_histories(mf, dt, out_dt, B, T, V, room):
    """The forms of more threads, the last of which takes more than 32 MiB of logits."""
    _logits(mf, B, T, V, dt, out_dt, room=room, n_bias=20, n_masks=3, drafts="tree" if T > 1 else None, lengths=[room - 5] * B, prompts=[room // 3] * B)


@pytest.mark.parametrize("dt,out_dt,in_place", [t + (False,) for t in TYPES] + [(torch.bfloat16, None, True), (torch.float32, None, True)])
@pytest.mark.parametrize("B,T,V,room", [(1600, 17, 504, 40), (1600, 17, 500, 41), (900, 5, 4504, 40), (320, 9, 1000, 3000), (320, 3, 8200, 2050),
                                        (70, 16, 700, 9000), (200, 17, 5200, 17000), (420, 2, 33000, 17000)])
def test_rows_that_share_a_block(mf, dt, out_dt, B, T, V, room, in_place):
    """With so many requests a block of threads has several rows of one, one after another; with one request a row each, to the same
    bits.  Masks of some rows, padded rows whose padding stays."""
    g = torch.Generator(device="cuda")
    g.manual_seed(B + T)

    def ids(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda").to(torch.int32)
    x = torch.randn((B, T, V + 8), generator=g, device="cuda").to(dt)
    a = dict(tokens=ids(-1, V + 9, B, room), lengths=ids(0, room + 1, B), prompt_lengths=ids(0, room // 2, B), drafts=ids(0, V // 4, B, T),
             tree=ids(0, 1 << (T - 1), B, T, 1), bias_ids=ids(0, V, B, 11), mask_rows=ids(-1, 6, B, T))
    a.update({n: 0.5 + torch.rand(shape, generator=g, device="cuda")
              for n, shape in (("repetition", (B,)), ("presence", (B,)), ("frequency", (B,)), ("bias", (B, 11)))})
    masks = ids(-2 ** 31, 2 ** 31, 5, (V + 31) // 32)
    out = x.clone() if in_place else torch.full((B, T, V + 8), 7.0, dtype=out_dt or dt, device="cuda")
    pad = out[..., V:].clone()
    mf.adjust_logits(out[..., :V] if in_place else x[..., :V], out[..., :V], masks=masks, **a)
    assert torch.equal(out[..., V:], pad)
    for b in sorted({0, 1, B // 3, B // 2, B - 2, B - 1}):
        one = torch.empty((1, T, V), dtype=out.dtype, device="cuda")
        mf.adjust_logits(x[b:b + 1, :, :V].contiguous(), one, masks=masks, **{n: t[b:b + 1] for n, t in a.items()})
        assert torch.equal(out[b, :, :V], one[0]), b


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_nothing_said_yet(mf, dt):
    """Histories with room for no token, and no masks, as tensors of such sizes: what is said has no part in the results."""
    none = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    zero, rows = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    x = torch.randn((2, 3, 1000), device="cuda").to(dt)
    drafts = torch.tensor([[5, 6, 7], [5, 5, 999]], dtype=torch.int32, device="cuda")
    f = torch.tensor([0.25, 0.5], device="cuda")
    for said in (dict(lengths=zero), dict(prompt_lengths=zero), dict(lengths=zero + 3, prompt_lengths=zero + 2), {}):
        for masked in ({}, dict(masks=torch.empty((0, 32), dtype=torch.int32, device="cuda"), mask_rows=rows)):
            for _ in range(2):
                a, b = torch.full_like(x, math.nan), torch.empty_like(x)
                mf.adjust_logits(x, a, tokens=none, frequency=f, drafts=drafts, **said, **masked)
                mf.adjust_logits(x, b, frequency=f, drafts=drafts)
                assert torch.equal(a, b) and not torch.equal(a, x)
    with pytest.raises(mf.MafatError):  # each row its mask, of none
        mf.adjust_logits(x, a, masks=torch.empty((0, 32), dtype=torch.int32, device="cuda"))
