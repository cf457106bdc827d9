"""The stride of a dimension of size one is nothing to go by: any is taken, as tensors cut from others have them."""
import pytest


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


# not a multiple of 16 bytes and below a head's channels, negative, past 2^40 bytes
ODD = [7, -3, (1 << 45) + 1]


@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("at", [0, 1, 2])
@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
def test_cross(mf, name, at, odd):
    sizes = [2, 3, 4]
    sizes[at] = 1
    strides = [2 * 3 * 4 * 64, 4 * 64, 64]
    strides[at] = odd
    tokens = {"n_q": sizes[1], "n_kv": 5} if name in ("q", "out") else {"n_q": 3, "n_kv": sizes[1]}
    mf.CrossAttention(batch=sizes[0], heads_q=sizes[2], heads_kv=sizes[2], head_dim=64, dry_run=True,
                      **tokens, **{name + "_strides": strides})


@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("name", ["prefix_k", "prefix_v", "own_k", "own_v"])
def test_prefix(mf, name, odd):
    for at in range(3):
        strides = [2 * 3 * 4 * 64, 4 * 64, 64]
        strides[at] = odd
        n = 1 if at == 1 else 3
        mf.PrefixAttention(prefixes=1 if at == 0 else 2, requests=1, n_q=1, n_prefix=n, n_own=n, heads_q=1 if at == 2 else 4,
                           heads_kv=1 if at == 2 else 4, head_dim=64, dry_run=True, **{name + "_strides": strides})


@pytest.mark.parametrize("odd", ODD)
def test_without_keys(mf, odd):
    """No room for keys: no stride of theirs is used."""
    mf.CrossAttention(2, 1, 0, 4, 4, 64, k_strides=(odd, odd, 64), v_strides=(512, odd, 64), dry_run=True)


def test_others_are_refused_as_before(mf):
    for strides in ((7, 256, 64), (-1024, 256, 64), (1 << 45, 256, 64), (1024, 60, 64), (0, 256, 64)):
        with pytest.raises(mf.MafatError):
            mf.CrossAttention(2, 1, 5, 4, 4, 64, k_strides=strides, dry_run=True)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 140])
@pytest.mark.parametrize("dtype", [0, 1])
def test_runs_with_them(mf, dtype, T):
    """One sequence of one key head, cut from larger tensors: the same results as from packed ones."""
    torch = pytest.importorskip("torch")
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    dt = (torch.bfloat16, torch.float32)[dtype]
    q, k, v = (torch.randn(s, generator=g, device="cuda").to(dt) for s in ((1, T, 4, 64), (1, 300, 1, 64), (1, 300, 1, 64)))
    o = [torch.empty_like(q) for _ in range(2)]
    mf.CrossAttention(1, T, 300, 4, 1, 64, dtype=dtype).run(q, k, v, o[0])
    odd = dict(q_strides=(7, 256, 64), k_strides=((1 << 45) + 1, 64, 5), v_strides=(3, 64, (1 << 45) + 1), out_strides=(9, 256, 64))
    q, k, v, out = (torch.as_strided(t, t.shape, s + (1,)) for t, s in zip((q, k, v, o[1]), odd.values()))
    mf.CrossAttention(1, T, 300, 4, 1, 64, dtype=dtype, **odd).run(q, k, v, out)
    assert torch.equal(o[0], o[1])
