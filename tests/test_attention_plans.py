"""Attention plans without a GPU: what is refused, and what a dry run says."""
import ctypes
import math

import pytest


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


CROSS = dict(batch=2, n_q=3, n_kv=100, heads_q=8, heads_kv=2, head_dim=64, dry_run=True)
PREFIX = dict(prefixes=2, requests=3, n_q=1, n_prefix=100, n_own=20, heads_q=8, heads_kv=2, head_dim=64, dry_run=True)


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), "EINVAL"), (dict(n_q=0), "EINVAL"), (dict(n_kv=-1), "EINVAL"), (dict(heads_kv=3), "EINVAL"),
    (dict(heads_q=0), "EINVAL"), (dict(heads_kv=0), "EINVAL"), (dict(head_dim=0), "EINVAL"), (dict(head_dim=12), "EUNSUPPORTED"),
    (dict(head_dim=136), "EUNSUPPORTED"), (dict(dtype=2), "EINVAL"), (dict(scale=-1.0), "EINVAL"), (dict(scale=math.inf), "EINVAL"),
    (dict(scale=math.nan), "EINVAL"), (dict(kernel=3), "EINVAL"), (dict(splits=-1), "EINVAL"), (dict(splits=129), "EINVAL"),
    (dict(k_strides=(12800, 128, 60)), "EINVAL"), (dict(k_strides=(12800, 0, 64)), "EINVAL"), (dict(v_strides=(12804, 128, 64)), "EINVAL"),
    (dict(q_strides=(-1536, 512, 64)), "EINVAL"), (dict(v_strides=(1 << 41, 128, 64)), "EUNSUPPORTED"),
    (dict(out_strides=(512, 512, 64)), "EINVAL"), (dict(batch=1 << 20, n_q=1 << 20), "EUNSUPPORTED")])
def test_cross_refusals(mf, change, status):
    with pytest.raises(mf.MafatError) as e:
        mf.CrossAttention(**{**CROSS, **change})
    assert mf.STATUS[e.value.status] == status, str(e.value)


@pytest.mark.parametrize("change,status", [
    (dict(prefixes=0), "EINVAL"), (dict(requests=0), "EINVAL"), (dict(n_prefix=-1), "EINVAL"), (dict(n_own=-5), "EINVAL"),
    (dict(n_q=0), "EINVAL"), (dict(heads_q=7), "EINVAL"), (dict(head_dim=20), "EUNSUPPORTED"),
    (dict(prefixes=1 << 20, requests=1 << 20), "EUNSUPPORTED"), (dict(own_k_strides=(2560, 64, 60)), "EINVAL"),
    (dict(prefix_v_strides=(12800, 130, 64)), "EINVAL")])
def test_prefix_refusals(mf, change, status):
    with pytest.raises(mf.MafatError) as e:
        mf.PrefixAttention(**{**PREFIX, **change})
    assert mf.STATUS[e.value.status] == status, str(e.value)


def test_struct_size_and_null_arguments(mf):
    h = ctypes.c_void_p()
    for desc, plan in ((mf.CrossDesc(), mf.lib.mafat_cross_plan), (mf.PrefixDesc(), mf.lib.mafat_prefix_plan)):
        assert plan(ctypes.byref(desc), ctypes.byref(h)) == mf.EINVAL
        assert plan(None, ctypes.byref(h)) == mf.EINVAL
        assert plan(ctypes.byref(desc), None) == mf.EINVAL
    assert mf.lib.mafat_rms_norm(None, *[None] * 7) == mf.EINVAL
    assert mf.lib.mafat_rms_norm(ctypes.byref(mf.NormDesc()), *[None] * 7) == mf.EINVAL
    assert mf.lib.mafat_cross_run(*[None] * 9) == mf.EINVAL
    assert mf.lib.mafat_prefix_run(*[None] * 12) == mf.EINVAL
    assert mf.lib.mafat_attn_stats(None, None) == mf.EINVAL
    assert mf.lib.mafat_attn_sync_status(None, None) == mf.EINVAL
    mf.lib.mafat_attn_destroy(None)


def test_dry_runs_are_not_run(mf):
    plan = mf.CrossAttention(**CROSS)
    with pytest.raises(mf.MafatError) as e:
        plan.run(4096, 8192, 16384, 32768)
    assert e.value.status == mf.EINVAL and "dry_run" in str(e.value)
    with pytest.raises(mf.MafatError):
        plan.sync_status()
    other = mf.PrefixAttention(**PREFIX)
    assert mf.lib.mafat_cross_run(other.handle, *[4096] * 8) == mf.EINVAL
    assert mf.lib.mafat_prefix_run(plan.handle, *[4096] * 11) == mf.EINVAL


@pytest.mark.parametrize("dtype", [0, 1])
def test_splits_cover_the_keys_and_the_workspace_their_parts(mf, dtype):
    for n_kv in (0, 1, 64, 65, 1444, 100000):
        for n_q in (1, 5, 700):
            for splits in (0, 1, 7, 128):
                s = mf.CrossAttention(**{**CROSS, "n_kv": n_kv, "n_q": n_q, "splits": splits, "dtype": dtype}).stats()
                assert 1 <= s["splits"][0] <= mf.MAX_SPLITS
                # a cluster of CTAs joins the parts of a small call without the workspace
                assert s["parts"] == s["splits"][0] or (splits == 0 and s["parts"] == 1 and s["splits"][0] in (2, 4, 8))
                assert s["launches_per_run"] == (1 if s["parts"] == 1 else 2)
                rows = 2 * n_q * 8
                assert s["workspace_bytes"] >= (rows * s["parts"] * (64 + 1) * 4 if s["parts"] > 1 else 0)


def test_the_second_launch_joins_the_parts_where_it_has_whole_rows(mf):
    s = mf.PrefixAttention(**PREFIX).stats()
    assert s["splits"][1] == 1 and s["parts"] == s["splits"][0] and s["launches_per_run"] == 2
    assert s["workspace_bytes"] >= 6 * 8 * s["parts"] * 65 * 4
    s = mf.PrefixAttention(**{**PREFIX, "n_own": 20000, "splits": 5}).stats()
    assert s["splits"] == [2, 5] and s["parts"] == 7 and s["launches_per_run"] == 3
    for empty, used in (("n_own", 0), ("n_prefix", 1)):
        s = mf.PrefixAttention(**{**PREFIX, empty: 0, "splits": 1}).stats()
        assert s["parts"] == 1 and s["launches_per_run"] == 1 and s["ctas"][used] > 0 and s["ctas"][1 - used] == 0
    s = mf.PrefixAttention(**{**PREFIX, "n_own": 0, "n_prefix": 0}).stats()
    assert s["parts"] == 1 and s["launches_per_run"] == 1


def test_a_single_sequence_may_have_any_stride_where_it_is_not_used(mf):
    mf.CrossAttention(1, 1, 100, 8, 2, 64, q_strides=(0, 0, 64), k_strides=(0, 128, 64), dry_run=True)
