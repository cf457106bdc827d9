"""Where rotary positions take tensors that lie between one another: by which elements they have, not by where they begin and end."""
import ctypes
import itertools
import random

import pytest

import fake_device

B, T, H, D = 2, 3, 2, 16  # sequences, tokens, heads, channels
BASE = 1 << 36


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


@pytest.fixture(scope="module")
def fake(mf, tmp_path_factory):
    return fake_device.build(mf, str(tmp_path_factory.mktemp("fake")))


@pytest.fixture(scope="module")
def plan(mf, fake):
    d, h = mf.RotaryDesc(struct_size=ctypes.sizeof(mf.RotaryDesc), head_dim=D), ctypes.c_void_p()
    assert fake.lib.mafat_rotary_plan(ctypes.byref(d), ctypes.byref(h)) == mf.OK
    return h


def _run(mf, fake, plan, tensors, places=None, room=T):
    """tensors: name -> (offset in elements, strides)."""
    c = mf.RotaryCall(struct_size=ctypes.sizeof(mf.RotaryCall), batch=B, n_q=T, heads_q=H, heads_kv=H, room=room)
    names = ("q", "q_out", "k", "k_out", "v", "v_out")
    a = []
    for n in names:
        a.append(BASE + 2 * tensors[n][0] if n in tensors else None)
        if n in tensors:
            getattr(c, n + "_strides")[:] = tensors[n][1]
    return fake.lib.mafat_rotary_run(plan, ctypes.byref(c), 1 << 32, places, *a, None)


def _packed(order, sizes):
    """Strides by the order of the dimensions, the last innermost; channels inside it."""
    st, step = {}, D
    for d in reversed(order):
        st[d], step = step, step * sizes[d]
    return st, step


@pytest.mark.parametrize("order", list(itertools.permutations("bwth")))
@pytest.mark.parametrize("room", [T, 5])
def test_keys_and_values_of_one_cache(mf, fake, plan, order, room):
    """[batch], keys or values, [place] and [head] in any order."""
    st, size = _packed(order, dict(b=B, w=2, t=room, h=H))
    strides = (st["b"], st["t"], st["h"])
    far = (T * H * D, H * D, D)
    tensors = dict(k=(1 << 20, far), v=(1 << 21, far), k_out=(0, strides), v_out=(st["w"], strides))
    assert _run(mf, fake, plan, tensors, places=(1 << 32) + 4096, room=room) == mf.OK, fake.lib.mafat_last_error()
    tensors["v_out"] = (st["w"] - 8, strides)  # half a head into the keys
    assert _run(mf, fake, plan, tensors, places=(1 << 32) + 4096, room=room) == mf.EINVAL
    assert fake.lib.mafat_last_error() == b"an output overlaps another tensor"


@pytest.mark.parametrize("order", list(itertools.permutations("bwth")))
def test_in_place_beside_others(mf, fake, plan, order):
    """Queries, keys and values of one matrix in any order, queries and keys turned where they are."""
    st, _ = _packed(order, dict(b=B, w=3, t=T, h=H))
    q, k, v = ((i * st["w"], (st["b"], st["t"], st["h"])) for i in range(3))
    assert _run(mf, fake, plan, dict(q=q, q_out=q, k=k, k_out=k, v=v, v_out=(1 << 20, (T * H * D, H * D, D)))) == mf.OK, fake.lib.mafat_last_error()


def test_what_is_taken_shares_no_element(mf, fake, plan):
    """Of random layouts: those that are taken write no element twice and none that is read elsewhere."""
    rng = random.Random(4)
    sizes = (B, T, H)

    def layout():
        order, st, step = rng.sample(range(3), 3), [0] * 3, D
        for d in order:
            st[d] = step + 8 * rng.choice([0, 0, 0, 1, 2, 5, 2 * H, 2 * T * H])
            step = st[d] * sizes[d]
        return 8 * rng.randrange(0, 40), tuple(st)

    def elements(t):  # in runs of 8
        return {(t[0] + sum(i * s for i, s in zip(at, t[1]))) // 8 + c for at in itertools.product(*map(range, sizes)) for c in range(D // 8)}
    taken = 0
    for _ in range(4000):
        q, q_out, k = layout(), layout(), layout()
        if rng.random() < 0.5:
            k = (8 * rng.randrange(0, 40), q_out[1])
        ok = _run(mf, fake, plan, dict(q=(q[0] + (1 << 20), q[1]), q_out=q_out, k=k, k_out=(1 << 21, (T * H * D, H * D, D)))) == mf.OK
        if ok:
            taken += 1
            assert not elements(q_out) & elements(k), (q_out, k)
    assert taken > 50, taken
