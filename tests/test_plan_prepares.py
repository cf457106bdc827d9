"""A plan prepares the kernels that it can launch and no others."""
import ctypes

import pytest

import fake_device


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


@pytest.fixture(scope="module")
def fake(mf, tmp_path_factory):
    return fake_device.build(mf, str(tmp_path_factory.mktemp("fake")))


@pytest.mark.parametrize("kind", ["cross", "prefix", "tree"])
@pytest.mark.parametrize("dtype", ["BF16", "FP32"])
@pytest.mark.parametrize("dim", [40, 128])
@pytest.mark.parametrize("keys", [0, 700])
def test_plans(mf, fake, kind, dtype, dim, keys):
    h = ctypes.c_void_p()
    common = dict(dtype=getattr(mf, dtype), n_q=4, heads_q=8, heads_kv=4, head_dim=dim)
    if kind == "cross":
        d = mf.CrossDesc(struct_size=ctypes.sizeof(mf.CrossDesc), batch=2, n_kv=keys, **common)
    else:
        d = mf.PrefixDesc(struct_size=ctypes.sizeof(mf.PrefixDesc), prefixes=2, requests=3, n_prefix=keys, n_own=20, **common)
    fake.reset()
    assert getattr(fake.lib, "mafat_%s_plan" % kind)(ctypes.byref(d), ctypes.byref(h)) == mf.OK
    of = " %d %d" % (kind == "tree", dim)
    assert [n for n in fake.notes() if n.startswith("prepare")] == ["prepare " + n + of for n in (("simt",) if dtype == "FP32" else ("rows", "tc"))]
    fake.lib.mafat_attn_destroy(h)


@pytest.mark.parametrize("call,dtype", [("prepare simt", "FP32"), ("prepare rows", "BF16"), ("prepare tc", "BF16")])
def test_kernels_that_cannot_be_prepared(mf, fake, call, dtype):
    h = ctypes.c_void_p()
    d = mf.CrossDesc(struct_size=ctypes.sizeof(mf.CrossDesc), batch=2, n_kv=100, n_q=4, heads_q=8, heads_kv=4, head_dim=64,
                     dtype=getattr(mf, dtype))
    fake.reset()
    fake.fail(call)
    assert mf.STATUS[fake.lib.mafat_cross_plan(ctypes.byref(d), ctypes.byref(h))] == "ECUDA" and not h.value
