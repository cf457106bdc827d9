"""Attention of drafted tokens, a tree for each request, against its definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from draft_util import random_ways, seen_own, words  # noqa: E402
from lm_util import attention64, attention_tol, check, check_lse, lse_tol  # noqa: E402


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _tree(mf, G, R, T, P, S, H, Hk, D, dtype, nodes=None, own_len=None, prefix_len=None, prefix_mask=None, shared=False,
          kernel=0, splits=0, scale=0.0, seed=1, poison=False, layout="packed", repeat=1, ways=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, dt = G * R, torch.bfloat16 if dtype == mf.BF16 else torch.float32

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)
    q, pk, pv, ok, ov = randn(n, T, H, D), randn(G, P, Hk, D), randn(G, P, Hk, D), randn(n, S, Hk, D), randn(n, S, Hk, D)
    lens = [min(S, T + (7 * b) % max(1, S - T + 1)) for b in range(n)] if own_len is None else own_len
    counts = [T] * n if nodes is None else nodes
    way = (random_ways(1, T, seed).expand(n, T, T) if shared else random_ways(n, T, seed)) if ways is None else ways
    seen_p = torch.ones(G, P, dtype=torch.bool)
    if prefix_len is not None:
        seen_p &= torch.arange(P)[None] < torch.tensor(prefix_len)[:, None]
    if prefix_mask is not None:
        seen_p &= prefix_mask
    seen_o = torch.stack([seen_own(way[b], lens[b], counts[b], T, S) for b in range(n)])
    if poison:  # what no query may read
        bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda")

        def spoil(x, seen):
            fill = bad[torch.arange(x.shape[1] * D, device="cuda") % 3].view(1, x.shape[1], 1, D).to(dt)
            return torch.where(seen.cuda()[:, :, None, None], x, fill)
        readable = torch.arange(S)[None] < torch.tensor(lens).clamp(0, S)[:, None]
        pk, pv, ok, ov = spoil(pk, seen_p), spoil(pv, seen_p), spoil(ok, readable), spoil(ov, readable)
        q[torch.arange(T)[None].cuda() >= torch.tensor(counts).cuda()[:, None]] = math.nan  # of places without a node
    kw = {}
    o = torch.full((n, T, H, D), math.nan, dtype=dt, device="cuda")
    if layout == "side":  # queries, keys and values of the caches in wider rows
        def put(x, wider):
            b = torch.full(x.shape[:2] + (x.shape[2] + wider, D + 8), math.nan, dtype=dt, device="cuda")[:, :, 1:x.shape[2] + 1, :D]
            return b.copy_(x)
        q, pk, pv, ok, ov, o = put(q, 2), put(pk, 1), put(pv, 2), put(ok, 3), put(ov, 1), put(o, 2)
        kw = {"q_strides": q.stride()[:3], "prefix_k_strides": pk.stride()[:3], "prefix_v_strides": pv.stride()[:3],
              "own_k_strides": ok.stride()[:3], "own_v_strides": ov.stride()[:3], "out_strides": o.stride()[:3]}
    lse = torch.full((n, T, H), math.nan, device="cuda")
    plan = mf.TreeAttention(G, R, T, P, S, H, Hk, D, dtype=dtype, scale=scale, kernel=kernel, splits=splits, **kw)

    def ints(x):
        return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    for _ in range(repeat):
        plan.run(q, pk, pv, ok, ov, words(way[:1] if shared else way).cuda(), o, nodes=ints(nodes), prefix_len=ints(prefix_len),
                 prefix_mask=None if prefix_mask is None else prefix_mask.cuda(), own_len=ints(lens), lse=lse)
    plan.sync_status(like=q)
    sc = scale or 1 / math.sqrt(D)
    for b in range(n):
        live = torch.arange(T, device="cuda") < counts[b]
        segs = [(pk[b // R], pv[b // R], seen_p[b // R].cuda()[None] & live[:, None]), (ok[b], ov[b], seen_o[b].cuda())]
        ref, rl, a, mag = attention64(q[b], segs, sc)
        check(o[b], ref, attention_tol(ref, a, mag, P + S, D, dtype == mf.BF16), "out %d" % b)
        check_lse(lse[b], rl, lse_tol(rl, mag, P + S, D), "lse %d" % b)
        assert not o[b][~live].any()
    return o, lse, plan


KERNELS = [0, 1, 2]
TYPES = [0, 1]


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,R,T,P,S,H,Hk,D", [
    (1, 1, 1, 1, 1, 1, 1, 64), (1, 1, 8, 196, 20, 8, 4, 64), (2, 3, 5, 130, 40, 4, 4, 128), (1, 2, 31, 64, 31, 2, 1, 40),
    (1, 2, 32, 257, 33, 4, 2, 64), (2, 1, 33, 100, 140, 8, 2, 72), (1, 3, 64, 128, 65, 2, 2, 128), (1, 1, 65, 300, 200, 8, 1, 64),
    (1, 2, 129, 70, 400, 2, 1, 128), (3, 2, 17, 1000, 129, 6, 2, 112), (1, 2, 100, 33, 100, 16, 2, 8)])
def test_sizes(mf, kernel, dtype, G, R, T, P, S, H, Hk, D):
    _tree(mf, G, R, T, P, S, H, Hk, D, dtype, kernel=kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("splits", [0, 1, 3, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_ragged_trees_and_lengths(mf, kernel, dtype, splits, D):
    """No node, one, all and more than there is room for; own keys fewer than nodes, none, and past the room; prefixes of
    no key and one.  Unread places hold NaN and infinities."""
    _tree(mf, 3, 3, 37, 150, 90, 4, 2, D, dtype, nodes=[0, 1, 37, 99, -3, 20, 36, 37, 5], own_len=[90, 1, 20, 200, 10, 0, 64, 37, 70],
          prefix_len=[0, 1, 999], kernel=kernel, splits=splits, poison=True, repeat=2)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_read_nothing(mf, kernel, dtype):
    """Trees whose bits are all zero, with no key before them."""
    way = torch.zeros(4, 6, 6, dtype=torch.bool)
    way[1, 2, 1] = way[2, 5, 5] = True
    _tree(mf, 2, 2, 6, 10, 40, 4, 2, 64, dtype, prefix_len=[0, 3], own_len=[6, 6, 6, 20], nodes=[6, 6, 6, 6], kernel=kernel, ways=way)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [3, 40, 96])
def test_one_set_of_keys(mf, kernel, dtype, T):
    """Without a prefix, and without room for own keys."""
    _tree(mf, 2, 2, T, 0, T + 90, 4, 2, 64, dtype, kernel=kernel, nodes=[T, 1, T - 1, 2])
    _tree(mf, 2, 2, T, 300, 0, 4, 2, 64, dtype, kernel=kernel, nodes=[T, 1, 0, 2], own_len=[0] * 4)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D", [(7, 64), (70, 128)])
def test_prefix_masks_and_shared_trees(mf, kernel, dtype, T, D):
    at = torch.arange(333)
    mask = torch.stack([at % 3 == 0, at < 0, (at >= 100) & (at < 228)])
    _tree(mf, 3, 2, T, 333, T + 50, 4, 2, D, dtype, prefix_mask=mask, prefix_len=[333, 333, 200], kernel=kernel, shared=True,
          nodes=[T, 3, T, 0, T - 1, T], poison=True)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [9, 50])
def test_strides_and_scale(mf, kernel, dtype, T):
    _tree(mf, 2, 2, T, 140, T + 30, 4, 2, 64, dtype, kernel=kernel, layout="side", scale=0.4, poison=True)


@pytest.mark.parametrize("D,H,Hk", [(128, 32, 8), (64, 16, 4)])
@pytest.mark.parametrize("T", [16, 61])
def test_many_requests(mf, D, H, Hk, T):
    """Prefixes read by tiles of many requests, and more work than the GPU holds at once."""
    n = 24
    _tree(mf, 2, n // 2, T, 2500, 260, H, Hk, D, mf.BF16, nodes=[1 + (11 * b) % T for b in range(n)], repeat=2, poison=True)


@pytest.mark.parametrize("first", [1, 31, 32, 33, 63, 64, 95, 96, 127, 128, 129, 200])
@pytest.mark.parametrize("kernel", KERNELS)
def test_trees_that_start_anywhere_in_a_tile(mf, first, kernel):
    _tree(mf, 1, 1, 70, 20, 300, 4, 1, 64, mf.BF16, own_len=[first + 70], kernel=kernel, poison=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kernel", KERNELS)
def test_a_chain_is_prefix_attention(mf, dtype, kernel):
    """A tree whose nodes follow one another: what PrefixAttention gives, to the bit where both have the same parts."""
    G, R, T, P, S, H, Hk, D = 2, 3, 20, 200, 60, 8, 2, 64
    chain = torch.ones(T, T, dtype=torch.bool).tril()[None].expand(G * R, T, T)
    o, lse, _ = _tree(mf, G, R, T, P, S, H, Hk, D, dtype, ways=chain, own_len=[60, 20, 33, 47, 59, 21], kernel=kernel, splits=1)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    dt = o.dtype
    q, pk, pv, ok, ov = [torch.randn(s, generator=g, device="cuda").to(dt) for s in
                         ((G * R, T, H, D), (G, P, Hk, D), (G, P, Hk, D), (G * R, S, Hk, D), (G * R, S, Hk, D))]
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    mf.PrefixAttention(G, R, T, P, S, H, Hk, D, dtype=dtype, kernel=kernel, splits=1).run(
        q, pk, pv, ok, ov, o2, own_len=torch.tensor([60, 20, 33, 47, 59, 21], dtype=torch.int32, device="cuda"), lse=lse2)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_results_repeat_on_other_streams(mf):
    """Two plans at once on two streams, and each again alone."""
    a = _tree(mf, 2, 4, 16, 3000, 100, 16, 4, 64, mf.BF16, seed=3)[0]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(_tree(mf, 2, 4, 16, 3000, 100, 16, 4, 64, mf.BF16, seed=3)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, x) for x in got)


def test_empty_and_wide_trees_of_one_request(mf):
    """More nodes than one tile of rows has, with one head for all."""
    _tree(mf, 1, 1, 300, 129, 500, 3, 1, 64, mf.BF16)
    _tree(mf, 1, 1, 300, 129, 500, 2, 1, 64, mf.FP32, nodes=[257])


@pytest.mark.parametrize("D,P,lens", [(128, 12000, [12000, 12000]), (128, 12000, [9999, 300]), (64, 9000, [0, 1]), (64, 9000, [8000, 127])])
def test_keys_that_idle_sms_take(mf, D, P, lens):
    """Prefixes whose tiles leave SMs idle: two parts of unequal length, also of sequences shorter than the first."""
    o, _, plan = _tree(mf, 2, 32, 16, P, 100, 32, 8, D, mf.BF16, prefix_len=lens, nodes=[1 + (5 * b) % 16 for b in range(64)], poison=True)
    s = plan.stats()
    assert s["splits"][0] == 2 and s["ctas"][0] % 2 == 0 and s["ctas"][0] // 2 < 152


@pytest.mark.parametrize("G,R,T,P,S,H,Hk,D", [(8, 30, 1, 50, 40, 8, 2, 64), (4, 13, 2, 18, 8, 8, 8, 128), (4, 27, 4, 105, 10, 16, 4, 128), (6, 33, 4, 17, 24, 4, 2, 72)])
def test_many_short_items(mf, G, R, T, P, S, H, Hk, D):
    """One launch of CTAs that take several items, each over both sets of keys; sets of every length, also of none."""
    n = G * R
    assert mf.TreeAttention(G, R, T, P, S, H, Hk, D, dry_run=True).stats()["whole_ctas"] == 304
    _tree(mf, G, R, T, P, S, H, Hk, D, mf.BF16, own_len=[(11 * b) % (S + 2) for b in range(n)], prefix_len=[(P * g) // (G - 1) for g in range(G)],
          nodes=[(3 * b) % (T + 1) for b in range(n)], poison=True, repeat=2)
    _tree(mf, G, R, T, P, S, H, Hk, D, mf.BF16, poison=True)
