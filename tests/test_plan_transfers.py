"""A plan is whole on the device when its maker returns: what was copied or set for it has been waited for, so that a run on any
stream, also one that the legacy stream does not hold up, finds it."""
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


def _is_whole(notes):
    sent = [i for i, n in enumerate(notes) if n in ("copy in", "set")]
    assert sent, notes
    assert "sync 0" in notes[sent[-1] + 1:], notes


def _rotary(mf, fake):
    d = mf.RotaryDesc(struct_size=ctypes.sizeof(mf.RotaryDesc), head_dim=64)
    h = ctypes.c_void_p()
    return fake.lib.mafat_rotary_plan(ctypes.byref(d), ctypes.byref(h)), h


def test_rotary_plan(mf, fake):
    fake.reset()
    status, h = _rotary(mf, fake)
    assert status == mf.OK
    _is_whole(fake.notes())
    fake.lib.mafat_rotary_destroy(h)


def test_rotary_plan_whose_transfer_fails(mf, fake):
    for call in ("copy in", "sync"):
        fake.reset()
        fake.fail(call)
        status, h = _rotary(mf, fake)
        assert mf.STATUS[status] == "ECUDA" and not h.value
        assert fake.notes().count("malloc") == fake.notes().count("free") == 1


def _attention(mf, fake, kind):
    h = ctypes.c_void_p()
    if kind == "cross":
        d = mf.CrossDesc(struct_size=ctypes.sizeof(mf.CrossDesc), batch=2, n_q=1, n_kv=100, heads_q=8, heads_kv=4, head_dim=64)
        return fake.lib.mafat_cross_plan(ctypes.byref(d), ctypes.byref(h)), h
    d = mf.PrefixDesc(struct_size=ctypes.sizeof(mf.PrefixDesc), prefixes=2, requests=3, n_q=4, n_prefix=100, n_own=20, heads_q=8,
                      heads_kv=4, head_dim=64)
    return getattr(fake.lib, "mafat_%s_plan" % kind)(ctypes.byref(d), ctypes.byref(h)), h


@pytest.mark.parametrize("kind", ["cross", "prefix", "tree"])
def test_attention_plans(mf, fake, kind):
    fake.reset()
    status, h = _attention(mf, fake, kind)
    assert status == mf.OK
    _is_whole(fake.notes())
    fake.lib.mafat_attn_destroy(h)


@pytest.mark.parametrize("call", ["set", "sync"])
def test_attention_plan_whose_transfer_fails(mf, fake, call):
    fake.reset()
    fake.fail(call)
    status, h = _attention(mf, fake, "tree")
    assert mf.STATUS[status] == "ECUDA" and not h.value
    assert fake.notes().count("malloc") == fake.notes().count("free") == 1


def test_a_status_that_is_read_is_cleared_when_the_call_returns(mf, fake):
    status, h = _attention(mf, fake, "cross")
    assert status == mf.OK
    fake.reset()
    assert fake.lib.mafat_attn_sync_status(h, None) == mf.OK and "set" not in fake.notes()
    fake.lib.fake_next_out(5)  # the next copy to the host brings this word
    fake.reset()
    assert mf.STATUS[fake.lib.mafat_attn_sync_status(h, None)] == "EDEVICE"
    _is_whole(fake.notes())
    fake.lib.mafat_attn_destroy(h)


LAYERS = [("conv", 3, 1, 1, 8), ("max", 2, 2, 0, 0), ("conv", 3, 1, 1, 16)]


def _network(mf, fake, dtype):
    net, h = ctypes.c_void_p(), ctypes.c_void_p()
    arr = mf.layer_descs(LAYERS)
    assert fake.lib.mafat_describe_net(arr, len(arr), 32, 32, 3, ctypes.byref(net)) == mf.OK
    c_in = 3
    for layer, (kind, k, _, _, filters) in enumerate(LAYERS):
        if kind == "conv":
            w, one = (ctypes.c_float * (filters * c_in * k * k))(), (ctypes.c_float * filters)()
            assert fake.lib.mafat_set_weights(net, layer, w, one, one) == mf.OK
            c_in = filters
    i32 = ctypes.c_int32 * 1
    status = fake.lib.mafat_plan(net, 1, None, i32(2), i32(2), 1, dtype, ctypes.byref(h))
    return status, net, h


@pytest.mark.parametrize("dtype", ["BF16", "FP32"])
def test_plans_of_networks(mf, fake, dtype):
    fake.reset()
    status, net, h = _network(mf, fake, getattr(mf, dtype))
    assert status == mf.OK, fake.lib.mafat_last_error()
    _is_whole(fake.notes())
    fake.reset()
    fake.lib.fake_next_out(5)
    assert fake.lib.mafat_sync_status(h, None) not in (mf.OK, mf.EINVAL)
    _is_whole(fake.notes())
    fake.lib.mafat_plan_destroy(h)
    fake.lib.mafat_net_destroy(net)


def test_a_plan_of_a_network_whose_transfer_fails(mf, fake):
    fake.reset()
    fake.fail("sync")
    status, net, h = _network(mf, fake, mf.FP32)
    assert mf.STATUS[status] == "ECUDA" and not h.value
    assert fake.notes().count("malloc") == fake.notes().count("free")
    fake.lib.mafat_net_destroy(net)


def test_the_area_of_calls_that_allocate_nothing(mf, fake):
    """Its status word is cleared by the device's first call, which another stream's run may follow."""
    status, net, h = _network(mf, fake, mf.FP32)
    assert status == mf.OK
    for first in (True, False):
        fake.reset()
        assert fake.lib.mafat_run_fp32_noalloc(h, 1 << 32, 1 << 33, None) == mf.OK
        notes = fake.notes()
        assert notes[:2] == ["set", "sync 0"] if first else "set" not in notes and "sync 0" not in notes, notes
    fake.lib.mafat_plan_destroy(h)
    fake.lib.mafat_net_destroy(net)
    fake.reset()
    assert fake.lib.mafat_noalloc_sync_status(None) == mf.OK and "set" not in fake.notes()
    fake.lib.fake_next_out(5)
    assert mf.STATUS[fake.lib.mafat_noalloc_sync_status(None)] == "EDEVICE"
    _is_whole(fake.notes())
