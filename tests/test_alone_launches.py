"""Which launches ask for their SMs alone, so that other streams' find no room there: none but fp32 tiles of 64 rows that are fewer than the
SMs and do not run beside the launch before."""
import ctypes
import re

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


AT = [(i + 1) << 36 for i in range(8)]


def _cross(mf, fake, batch, n_q, n_kv, heads, dim, dtype):
    d = mf.CrossDesc(struct_size=ctypes.sizeof(mf.CrossDesc), dtype=dtype, batch=batch, n_q=n_q, n_kv=n_kv, heads_q=heads, heads_kv=heads,
                     head_dim=dim)
    h = ctypes.c_void_p()
    assert fake.lib.mafat_cross_plan(ctypes.byref(d), ctypes.byref(h)) == mf.OK
    fake.reset()
    assert fake.lib.mafat_cross_run(h, AT[0], AT[1], AT[2], None, None, AT[3], None, None) == mf.OK, fake.lib.mafat_last_error()
    fake.lib.mafat_attn_destroy(h)
    return [n for n in fake.notes() if n.startswith("launch")]


def _prefix(mf, fake, prefixes, requests, n_q, n_prefix, n_own, heads_q, heads_kv, dim, dtype):
    d = mf.PrefixDesc(struct_size=ctypes.sizeof(mf.PrefixDesc), dtype=dtype, prefixes=prefixes, requests=requests, n_q=n_q, n_prefix=n_prefix,
                      n_own=n_own, heads_q=heads_q, heads_kv=heads_kv, head_dim=dim)
    h = ctypes.c_void_p()
    assert fake.lib.mafat_prefix_plan(ctypes.byref(d), ctypes.byref(h)) == mf.OK
    fake.reset()
    assert fake.lib.mafat_prefix_run(h, AT[0], AT[1], AT[2], None, None, AT[3], AT[4], None, AT[5], None, None) == mf.OK
    fake.lib.mafat_attn_destroy(h)
    return [n for n in fake.notes() if n.startswith("launch")]


def _simt(note):
    return tuple(int(x) for x in re.fullmatch(r"launch simt (\d+), CTAs (\d+), alone (\d+)", note).groups())


@pytest.mark.parametrize("dim", [64, 128])
def test_cross_attention(mf, fake, dim):
    for batch, alone in ((18, 1), (19, 0), (38, 0)):  # 144, 152 and 304 CTAs of 152 SMs
        assert _simt(_cross(mf, fake, batch, 64, 676, 8, dim, mf.FP32)[0]) == (64, batch * 8, alone)
    assert all("simt" not in n for n in _cross(mf, fake, 18, 128, 676, 8, dim, mf.BF16))


def test_beside_another_launch(mf, fake):
    """The prefix's 144 CTAs are alone, the own keys' 84 are launched beside them; so are the 128 behind 448."""
    first, second = _prefix(mf, fake, 6, 7, 24, 13517, 40, 4, 2, 64, mf.FP32)[:2]
    assert _simt(first) == (64, 144, 1) and _simt(second) == (64, 84, 0)
    first, second = _prefix(mf, fake, 4, 8, 8, 5776, 200, 16, 4, 128, mf.FP32)[:2]
    assert _simt(first) == (64, 448, 0) and _simt(second) == (64, 128, 0)
