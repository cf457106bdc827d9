"""Cross attention and attention over shared prefixes against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from lm_util import attention64, attention_tol, check, check_lse, lse_tol  # noqa: E402


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _dt(mf, dtype):
    return torch.bfloat16 if dtype == mf.BF16 else torch.float32


def _randn(g, shape, dt, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def _cross(mf, B, T, S, H, Hk, D, dtype, kv_len=None, kv_mask=None, kernel=0, splits=0, scale=0.0, seed=1, poison=False,
           spread=1.0, layout="bshd", repeat=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dt(mf, dtype)
    q = _randn(g, (B, T, H, D), dt, spread)
    k, v = _randn(g, (B, S, Hk, D), dt, spread), _randn(g, (B, S, Hk, D), dt)
    seen = torch.ones(B, S, dtype=torch.bool, device="cuda")
    ln = None
    if kv_len is not None:
        ln = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
        seen &= torch.arange(S, device="cuda")[None] < ln[:, None]
    if kv_mask is not None:
        seen &= kv_mask
    if poison:
        bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda")
        fill = bad[torch.arange(S * D, device="cuda") % 3].view(1, S, 1, D).to(dt)
        k = torch.where(seen[:, :, None, None], k, fill)
        v = torch.where(seen[:, :, None, None], v, fill)
    kw = {}
    if layout == "bhsd":  # heads outside the tokens, in a larger buffer with rows of its own
        def put(t, n):
            b = torch.full((B, t.shape[2], n + 3, D + 8), math.nan, dtype=dt, device="cuda")
            u = b[:, :, 1:n + 1, :D].transpose(1, 2)
            u.copy_(t)
            return u
        q, k, v = put(q, T), put(k, S), put(v, S)
        o = torch.full((B, H, T + 2, D + 16), math.nan, dtype=dt, device="cuda")[:, :, :T, :D].transpose(1, 2)
        kw = {"q_strides": q.stride()[:3], "k_strides": k.stride()[:3], "v_strides": v.stride()[:3], "out_strides": o.stride()[:3]}
    else:
        o = torch.full((B, T, H, D), math.nan, dtype=dt, device="cuda")
    lse = torch.full((B, T, H), math.nan, dtype=torch.float32, device="cuda")
    plan = mf.CrossAttention(B, T, S, H, Hk, D, dtype=dtype, scale=scale, kernel=kernel, splits=splits, **kw)
    for _ in range(repeat):
        plan.run(q, k, v, o, kv_len=ln, kv_mask=kv_mask, lse=lse)
    plan.sync_status(like=q)
    sc = scale or 1 / math.sqrt(D)
    for b in range(B):
        ref, rl, a, mag = attention64(q[b], [(k[b], v[b], seen[b][None].expand(T, -1))], sc)
        check(o[b], ref, attention_tol(ref, a, mag, S, D, dtype == mf.BF16), "out %d" % b)
        check_lse(lse[b], rl, lse_tol(rl, mag, S, D), "lse %d" % b)
    return o, lse


KERNELS = [0, 1, 2]
TYPES = [0, 1]


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,S,H,Hk,D", [
    (1, 1, 1, 1, 1, 64), (1, 1, 196, 8, 4, 64), (3, 1, 333, 8, 1, 128), (2, 2, 127, 4, 4, 64), (1, 5, 128, 6, 2, 128),
    (2, 17, 129, 4, 2, 40), (1, 33, 64, 2, 2, 8), (1, 130, 257, 3, 1, 72), (2, 300, 511, 2, 1, 128), (1, 257, 65, 8, 2, 64),
    (2, 9, 1000, 16, 2, 112), (1, 1, 2311, 32, 2, 128)])
def test_cross_sizes(mf, kernel, dtype, B, T, S, H, Hk, D):
    _cross(mf, B, T, S, H, Hk, D, dtype, kernel=kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("splits", [1, 2, 5, 128])
@pytest.mark.parametrize("T", [1, 40])
def test_cross_lengths_and_splits(mf, kernel, dtype, splits, T):
    """Lengths of zero, one, around tiles of 64 and 128 and past the room; unread places hold NaN and infinities."""
    _cross(mf, 9, T, 400, 4, 2, 64, dtype, kv_len=[0, 1, 63, 64, 65, 128, 129, 400, 999], kernel=kernel, splits=splits, poison=True)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D", [(1, 128), (150, 128), (7, 64)])
def test_cross_masks(mf, kernel, dtype, T, D):
    """Padded maps: a rectangle is readable, a sequence with nothing, one with a single key; NaN elsewhere."""
    S, w = 500, 25
    at = torch.arange(S, device="cuda")
    mask = torch.stack([(at // w < 13) & (at % w < 11), at < 0, at == 499, at >= 250, at % 2 == 0])
    _cross(mf, 5, T, S, 4, 2, D, dtype, kv_mask=mask, kv_len=[500, 500, 500, 470, 301], kernel=kernel, poison=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("T,D", [(90, 128), (90, 64)])
def test_cross_sparse_masks(mf, dtype, splits, T, D):
    """Readable keys in numbers around a tile's, with gaps longer than what is looked at at once."""
    at = torch.arange(1500, device="cuda")
    mask = torch.stack([at % 23 == 22, (at >= 700) & (at < 764), (at >= 600) & (at < 729), (at < 64) | (at >= 1499), at % 200 < 65,
                        (at < 127) | ((at >= 500) & (at < 628)), at >= 0])
    _cross(mf, 7, T, 1500, 2, 1, D, dtype, kv_mask=mask, kv_len=[1500] * 6 + [1345], kernel=2, splits=splits, poison=True, repeat=2)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,Hk,D", [(100, 1, 8, 8, 64), (128, 3, 4, 4, 128), (129, 1, 4, 4, 64), (77, 70, 8, 8, 128), (2, 1400, 16, 16, 64)])
def test_cross_many_sequences(mf, kernel, dtype, B, T, H, Hk, D):
    """More work than the GPU holds at once: lengths of zero, equal ones, past the room."""
    ln = [(37 * i * i + 11 * i) % 300 for i in range(B)]
    ln[:2], ln[-2:] = [0, 400], [64, 64]
    _cross(mf, B, T, 290, H, Hk, D, dtype, kv_len=ln, kernel=kernel, poison=True, repeat=2)


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("D", [64, 40, 128, 96])
@pytest.mark.parametrize("T", [150, 256, 333, 385])
def test_cross_tiles_of_256_rows(mf, T, D, mask):
    """Work for all SMs in tiles of two slots, of which the last tile has one or both, and some rows of each."""
    B, S = 152 // (-(-T // 256)), 700
    plan = mf.CrossAttention(B, T, S, 1, 1, D)
    assert plan.stats()["ctas"][0] == B * (-(-T // 256)) * plan.stats()["splits"][0]
    at = torch.arange(S, device="cuda")
    kw = {"kv_mask": torch.stack([at % (2 + i % 5) > 0 for i in range(B)])} if mask else {}
    _cross(mf, B, T, S, 1, 1, D, mf.BF16, kv_len=[(97 * i + 300) % 760 for i in range(B)], poison=True, repeat=3, **kw)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
def test_cross_strides(mf, kernel, dtype):
    _cross(mf, 2, 37, 211, 6, 3, 56, dtype, kernel=kernel, layout="bhsd", kv_len=[211, 100])
    _cross(mf, 2, 1, 211, 6, 3, 128, dtype, kernel=kernel, layout="bhsd")


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 64])
def test_cross_large_scores(mf, kernel, dtype, T):
    """Scores far apart: the running maximum moves by hundreds, most weights vanish."""
    _cross(mf, 1, T, 700, 4, 2, 64, dtype, kernel=kernel, spread=6.0, scale=0.7)
    _cross(mf, 1, T, 700, 4, 2, 64, dtype, kernel=kernel, scale=1e-3)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 200])
def test_cross_rising_scores(mf, kernel, dtype, T):
    """Each tile's scores are above the ones before: every tile rescales what it has."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    dt, S, D = _dt(mf, dtype), 900, 64
    q = torch.ones(1, T, 2, D, device="cuda", dtype=dt)
    k = (torch.arange(S, device="cuda").float() / 40)[None, :, None, None].expand(1, S, 2, D).to(dt).contiguous()
    v = _randn(g, (1, S, 2, D), dt)
    o = torch.empty_like(q)
    plan = mf.CrossAttention(1, T, S, 2, 2, D, dtype=dtype, kernel=kernel, splits=1)
    plan.run(q, k, v, o)
    plan.sync_status(like=q)
    ref, _, a, mag = attention64(q[0], [(k[0], v[0], torch.ones(T, S, dtype=torch.bool, device="cuda"))], 1 / 8)
    check(o[0], ref, attention_tol(ref, a, mag, S, D, dtype == mf.BF16), "out")


@pytest.mark.parametrize("dtype", TYPES)
def test_cross_no_keys(mf, dtype):
    dt = _dt(mf, dtype)
    q = torch.ones(2, 3, 4, 64, device="cuda", dtype=dt)
    o, lse = torch.full_like(q, math.nan), torch.empty(2, 3, 4, device="cuda")
    k = torch.empty(2, 0, 2, 64, device="cuda", dtype=dt)
    mf.CrossAttention(2, 3, 0, 4, 2, 64, dtype=dtype).run(q, k, k, o, lse=lse)
    assert (o == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
def test_nan_in_readable_places_is_seen(mf, kernel, dtype):
    dt = _dt(mf, dtype)
    for T in (1, 150):
        q = torch.ones(1, T, 2, 64, device="cuda", dtype=dt)
        k = torch.ones(1, 300, 2, 64, device="cuda", dtype=dt)
        k[0, 200, 1, 3] = math.nan
        v = torch.ones_like(k)
        o = torch.zeros_like(q)
        mf.CrossAttention(1, T, 300, 2, 2, 64, dtype=dtype, kernel=kernel).run(q, k, v, o)
        assert torch.isnan(o[:, :, 1]).all() and torch.isfinite(o[:, :, 0]).all()


def test_cross_offsets_past_32_bits(mf):
    """Two sequences whose keys lie more than 2^32 elements apart, and a head stride past 2^31."""
    for kernel in KERNELS:
        S, D = 150, 64
        far = (1 << 32) + 4096
        buf = torch.empty(far + (1 << 31) + 64 + S * D, dtype=torch.bfloat16, device="cuda")
        k = torch.as_strided(buf, (2, S, 2, D), (far, D, (1 << 31) + 64, 1))
        g = torch.Generator(device="cuda")
        g.manual_seed(8)
        k.copy_(_randn(g, (2, S, 2, D), torch.bfloat16))
        for T in (1, 140):
            q, v = _randn(g, (2, T, 4, D), torch.bfloat16), _randn(g, (2, S, 2, D), torch.bfloat16)
            o = torch.empty_like(q)
            mf.CrossAttention(2, T, S, 4, 2, D, k_strides=k.stride()[:3], kernel=kernel).run(q, k, v, o)
            for b in range(2):
                ref, _, a, mag = attention64(q[b], [(k[b], v[b], torch.ones(T, S, dtype=torch.bool, device="cuda"))], 1 / 8)
                check(o[b], ref, attention_tol(ref, a, mag, S, D, True), "out")
        del buf, k
        torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 300])
def test_runs_are_repeatable_on_another_stream_and_in_a_graph(mf, dtype, T):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    dt = _dt(mf, dtype)
    q, k, v = (_randn(g, s, dt) for s in ((2, T, 8, 64), (2, 900, 2, 64), (2, 900, 2, 64)))
    o = [torch.empty_like(q) for _ in range(3)]
    plan = mf.CrossAttention(2, T, 900, 8, 2, 64, dtype=dtype)
    plan.run(q, k, v, o[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    plan.run(q, k, v, o[1], stream=s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run(q, k, v, o[2])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o[0], o[1]) and torch.equal(o[0], o[2])


# ---- shared prefixes ------------------------------------------------------------------------


def _prefix(mf, G, R, T, P, S, H, Hk, D, dtype, own_len=None, prefix_len=None, prefix_mask=None, kernel=0, splits=0,
            seed=1, poison=False, strided=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, N = _dt(mf, dtype), G * R
    q = _randn(g, (N, T, H, D), dt)
    pk, pv = _randn(g, (G, P, Hk, D), dt), _randn(g, (G, P, Hk, D), dt)
    ok, ov = _randn(g, (N, S, Hk, D), dt), _randn(g, (N, S, Hk, D), dt)
    pl = None if prefix_len is None else torch.tensor(prefix_len, dtype=torch.int32, device="cuda")
    ol = None if own_len is None else torch.tensor(own_len, dtype=torch.int32, device="cuda")
    pseen = torch.ones(G, P, dtype=torch.bool, device="cuda")
    if pl is not None:
        pseen &= torch.arange(P, device="cuda")[None] < pl[:, None]
    if prefix_mask is not None:
        pseen &= prefix_mask
    n_own = torch.full((N,), S, device="cuda") if ol is None else ol.clamp(0, S)
    oread = torch.arange(S, device="cuda")[None] < n_own[:, None]
    if poison:
        pk, pv = (torch.where(pseen[:, :, None, None], t, torch.full_like(t, math.nan)) for t in (pk, pv))
        ok, ov = (torch.where(oread[:, :, None, None], t, torch.full_like(t, math.inf)) for t in (ok, ov))
    kw = {}
    if strided:  # one cache [key/value][request][head][place][channel], the prefix in another
        cache = torch.full((2, N, Hk, S + 5, D), math.nan, dtype=dt, device="cuda")
        cache[0, :, :, :S], cache[1, :, :, :S] = ok.transpose(1, 2), ov.transpose(1, 2)
        ok, ov = cache[0, :, :, :S].transpose(1, 2), cache[1, :, :, :S].transpose(1, 2)
        both = torch.stack([pk, pv], 2)  # keys and values side by side
        pk, pv = both[:, :, 0], both[:, :, 1]
        kw = {n + "_strides": t.stride()[:3] for n, t in (("prefix_k", pk), ("prefix_v", pv), ("own_k", ok), ("own_v", ov))}
    o = torch.full((N, T, H, D), math.nan, dtype=dt, device="cuda")
    lse = torch.full((N, T, H), math.nan, device="cuda")
    plan = mf.PrefixAttention(G, R, T, P, S, H, Hk, D, dtype=dtype, kernel=kernel, splits=splits, **kw)
    plan.run(q, pk, pv, ok, ov, o, prefix_len=pl, prefix_mask=prefix_mask, own_len=ol, lse=lse)
    plan.sync_status(like=q)
    t = torch.arange(T, device="cuda")
    for n in range(N):
        f = n // R
        seen = torch.arange(S, device="cuda")[None] <= (n_own[n] - T + t)[:, None]
        ref, rl, a, mag = attention64(q[n], [(pk[f], pv[f], pseen[f][None].expand(T, -1)), (ok[n], ov[n], seen)], 1 / math.sqrt(D))
        check(o[n], ref, attention_tol(ref, a, mag, P + S, D, dtype == mf.BF16), "out %d" % n)
        check_lse(lse[n], rl, lse_tol(rl, mag, P + S, D), "lse %d" % n)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,R,T,P,S,H,Hk,D", [
    (1, 1, 1, 1, 1, 1, 1, 64), (1, 5, 1, 196, 33, 8, 4, 64), (2, 3, 1, 130, 7, 8, 1, 128), (1, 17, 1, 676, 129, 4, 4, 40),
    (2, 2, 5, 300, 70, 6, 2, 128), (1, 3, 61, 257, 200, 4, 1, 64), (3, 1, 130, 64, 130, 2, 2, 72), (1, 40, 1, 1444, 90, 16, 2, 128)])
def test_prefix_sizes(mf, kernel, dtype, G, R, T, P, S, H, Hk, D):
    _prefix(mf, G, R, T, P, S, H, Hk, D, dtype, kernel=kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("T", [1, 6])
def test_prefix_lengths(mf, kernel, dtype, splits, T):
    """Own lengths of zero (with nothing but the prefix, or nothing at all), below and above n_q, at and past the room."""
    mask = torch.ones(3, 150, dtype=torch.bool, device="cuda")
    mask[0, 40:90] = False
    mask[0, ::3] = False
    _prefix(mf, 3, 4, T, 150, 140, 4, 2, 64, dtype, own_len=[0, 1, 5, 6, 7, 64, 65, 0, 128, 129, 140, 900],
            prefix_len=[150, 0, 65], prefix_mask=mask, kernel=kernel, splits=splits, poison=True)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
def test_prefix_strides(mf, kernel, dtype):
    _prefix(mf, 2, 3, 1, 210, 45, 8, 2, 64, dtype, own_len=[45, 1, 9, 33, 2, 0], kernel=kernel, strided=True)
    _prefix(mf, 1, 2, 9, 99, 45, 4, 2, 128, dtype, own_len=[45, 20], kernel=kernel, strided=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_prefix_without_room(mf, dtype):
    """No own keys, or no prefix: what is left is plain attention to the other set."""
    _prefix(mf, 1, 3, 1, 77, 0, 4, 2, 64, dtype)
    _prefix(mf, 2, 2, 4, 0, 50, 4, 2, 64, dtype)


def test_tensors_that_are_not_the_plans_are_refused(mf):
    plan = mf.CrossAttention(2, 3, 50, 4, 2, 64)
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 50, 2, 64, dtype=torch.bfloat16, device="cuda")
    good = dict(q=q, k=k, v=k.clone(), out=torch.empty_like(q))
    plan.run(**good)
    bad = [dict(q=q.float()), dict(k=k[:, :49]), dict(v=k.cpu()), dict(out=torch.empty(2, 3, 4, 128, dtype=q.dtype, device="cuda")[..., ::2]),
           dict(kv_len=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(kv_mask=torch.zeros(2, 49, dtype=torch.bool, device="cuda")),
           dict(lse=torch.zeros(2, 4, 3, device="cuda")), dict(out=q), dict(k=k.transpose(0, 1).contiguous().transpose(0, 1))]
    for change in bad:
        with pytest.raises(mf.MafatError) as e:
            plan.run(**{**good, **change})
        assert e.value.status == mf.EINVAL
    torch.cuda.synchronize()


@pytest.mark.parametrize("seed", range(24))
def test_random_sizes(mf, seed):
    """Sizes, types, lengths, masks and layouts at random, whatever kernel they go to."""
    import random
    r = random.Random(seed)
    dtype, D, Hk = r.choice([0, 0, 1]), 8 * r.randint(1, 16), r.choice([1, 2, 3, 5])
    H = Hk * r.choice([1, 2, 4, 7, 8])
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if r.random() < 0.5:
        B, T, S = r.randint(1, 5), r.choice([1, 1, r.randint(2, 300)]), r.randint(1, 1500)
        ln = [r.randint(0, S) for _ in range(B)] if r.random() < 0.5 else None
        mask = torch.rand(B, S, generator=g, device="cuda") < r.random() if r.random() < 0.5 else None
        _cross(mf, B, T, S, H, Hk, D, dtype, kv_len=ln, kv_mask=mask, seed=seed, poison=True, layout=r.choice(["bshd", "bhsd"]))
    else:
        G, R, T = r.randint(1, 3), r.randint(1, 9), r.choice([1, 1, r.randint(2, 40)])
        P, S = r.randint(1, 900), r.randint(1, 300)
        own = [r.randint(0, S) for _ in range(G * R)]
        pl = [r.randint(0, P) for _ in range(G)] if r.random() < 0.5 else None
        mask = torch.rand(G, P, generator=g, device="cuda") < r.random() if r.random() < 0.5 else None
        _prefix(mf, G, R, T, P, S, H, Hk, D, dtype, own_len=own, prefix_len=pl, prefix_mask=mask, seed=seed, poison=True,
                strided=r.random() < 0.5)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_lse_and_with_raw_addresses(mf, dtype):
    """lse is optional; addresses are taken as they are given, and refused where they cannot be right."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    dt = _dt(mf, dtype)
    q, k, v = (_randn(g, s, dt) for s in ((2, 3, 4, 64), (2, 90, 2, 64), (2, 90, 2, 64)))
    o = [torch.empty_like(q) for _ in range(2)]
    plan = mf.CrossAttention(2, 3, 90, 4, 2, 64, dtype=dtype)
    plan.run(q, k, v, o[0])
    s = torch.cuda.current_stream().cuda_stream
    plan.run(q.data_ptr(), k.data_ptr(), v.data_ptr(), o[1].data_ptr(), stream=s)
    plan.sync_status(like=q)
    assert torch.equal(o[0], o[1])
    addresses = dict(q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), out=o[1].data_ptr())
    for name in addresses:
        for wrong in (0, addresses[name] + 2, addresses["out" if name != "out" else "k"]):
            with pytest.raises(mf.MafatError) as e:
                plan.run(**{**addresses, name: wrong}, stream=s)
            assert e.value.status == mf.EINVAL
    for name in ("kv_len", "lse"):
        with pytest.raises(mf.MafatError):
            plan.run(**addresses, **{name: o[1].data_ptr() + 1}, stream=s)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kernel", [1, 2])
def test_long_fp32_sums_round_as_sums_do(mf, kernel):
    """24000 keys of nearly equal weight in one part: O is a random walk of n terms, whose every addition rounds by
    2^-25 of it (root mean square, about), so 2^-25 sqrt(n / 2) of the result; twice that, and 1e-6 for the weights.
    A factor a tile that is not exactly 1 where the maximum stays would show as a drift of the weights."""
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    T, S, D = 6, 24000, 64
    q, k, v = (_randn(g, s, torch.float32) for s in ((1, T, 4, D), (1, S, 1, D), (1, S, 1, D)))
    k[0, 0] = 3 * q[0, 0, 0] / q[0, 0, 0].norm() ** 2 * 8 / 0.37  # the maximum comes first for one row
    o = torch.empty_like(q)
    plan = mf.CrossAttention(1, T, S, 4, 1, D, dtype=mf.FP32, kernel=kernel, splits=1, scale=0.37 / 8)
    plan.run(q, k, v, o)
    plan.sync_status(like=q)
    ref = attention64(q[0], [(k[0], v[0], torch.ones(T, S, dtype=torch.bool, device="cuda"))], 0.37 / 8)[0]
    off = ((o[0].double() - ref).square().mean() / ref.square().mean()).sqrt().item()
    assert off <= 2 * 2.0 ** -25 * math.sqrt(S / 2) + 1e-6, off


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("G,R,T,P,S,H,Hk,D", [
    (2, 5, 30, 150, 70, 8, 2, 64), (3, 2, 70, 128, 256, 8, 2, 128), (2, 3, 90, 40, 301, 4, 1, 80), (1, 2, 33, 300, 33, 8, 8, 128),
    (2, 3, 1, 100, 20, 8, 2, 64)])
def test_prefix_in_one_launch(mf, mask, G, R, T, P, S, H, Hk, D):
    """Both sets read by the same tiles of rows (with a mask of the prefix, by two launches): lengths of zero on either side
    and on both, below the tokens', around tiles, past the room."""
    plan = mf.PrefixAttention(G, R, T, P, S, H, Hk, D)
    assert plan.stats()["whole_ctas"] > 0
    lens = [S, 0, T - 1, min(S, 128), S + 5, max(0, T - 7), 1]
    pl = [P, 0, 129][:G]
    kw = {}
    if mask:
        at = torch.arange(P, device="cuda")
        kw["prefix_mask"] = torch.stack([at % 3 > 0, at < 0, at >= P // 2][:G])
    _prefix(mf, G, R, T, P, S, H, Hk, D, mf.BF16, prefix_len=pl, own_len=[lens[i % 7] for i in range(G * R)], poison=True, **kw)
