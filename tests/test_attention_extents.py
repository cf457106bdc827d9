"""Sizes and strides at the ends of what an attention plan takes; dry runs."""
import pytest


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


CROSS = dict(batch=1, n_q=1, n_kv=100, heads_q=1, heads_kv=1, head_dim=64, dry_run=True)
PREFIX = dict(prefixes=1, requests=1, n_q=1, n_prefix=100, n_own=20, heads_q=1, heads_kv=1, head_dim=64, dry_run=True)


def _refused(mf, make, kw):
    with pytest.raises(mf.MafatError) as e:
        make(**kw)
    assert mf.STATUS[e.value.status] == "EUNSUPPORTED", str(e.value)


FAR = 1 << 38  # elements; of 2 bytes within the largest stride


@pytest.mark.parametrize("change", [
    dict(n_kv=1 << 30, heads_q=1 << 28, heads_kv=1 << 28, head_dim=128),    # packed: 2^65 elements
    dict(batch=1 << 25, k_strides=(FAR, 64, 64)), dict(batch=1 << 25, v_strides=(FAR, 64, 64)),
    dict(batch=1 << 25, q_strides=(FAR, 64, 64)), dict(batch=1 << 25, out_strides=(FAR, 64, 64)),
    dict(batch=1 << 12, n_kv=1 << 24, k_strides=(64, FAR, 64)),
    # 2^61 bytes each way
    dict(batch=(1 << 22) + 1, n_kv=(1 << 22) + 1, heads_q=(1 << 4) + 1, heads_kv=(1 << 4) + 1, k_strides=(FAR, FAR, 64))])
def test_cross_extents_past_62_bits_are_refused(mf, change):
    _refused(mf, mf.CrossAttention, {**CROSS, **change})


@pytest.mark.parametrize("change", [
    dict(n_prefix=1 << 30, heads_q=1 << 28, heads_kv=1 << 28, head_dim=128),
    dict(n_own=1 << 30, heads_q=1 << 28, heads_kv=1 << 28, head_dim=128),
    dict(prefixes=1 << 25, prefix_k_strides=(FAR, 64, 64)), dict(prefixes=1 << 25, prefix_v_strides=(FAR, 64, 64)),
    dict(requests=1 << 25, own_k_strides=(FAR, 64, 64)), dict(prefixes=1 << 13, requests=1 << 12, own_v_strides=(FAR, 64, 64))])
def test_prefix_extents_past_62_bits_are_refused(mf, change):
    _refused(mf, mf.PrefixAttention, {**PREFIX, **change})


def test_large_extents_are_taken(mf):
    mf.CrossAttention(**{**CROSS, "batch": 1 << 20, "k_strides": (FAR, 64, 64), "out_strides": (FAR, 64, 64)})
    mf.CrossAttention(**{**CROSS, "n_kv": 1 << 22, "k_strides": (64, FAR, 64)})
    mf.PrefixAttention(**{**PREFIX, "requests": 1 << 20, "own_k_strides": (FAR, 64, 64)})
    mf.CrossAttention(**{**CROSS, "n_kv": 0, "batch": 1 << 20, "k_strides": (FAR, 64, 64)})
