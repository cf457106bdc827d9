"""The operators of a drafting decoder without a GPU: what the library refuses, what the binding hands on, what plans say.
Addresses are made up: a refused call reads none of them."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


AT = [(i + 1) << 32 for i in range(20)]  # far apart, aligned


def _status(mf, got, want):
    assert mf.STATUS[got] == want, mf.lib.mafat_last_error().decode()


# ---- norms around a block ---------------------------------------------------------------------


def _norm(mf, at=None, null=(), **change):
    d = mf.BlockNormDesc(struct_size=ctypes.sizeof(mf.BlockNormDesc), dtype=0, out_dtype=0, cols=256, rows=12, branch_scale=1.0,
                         residual_scale=1.0, eps=1e-6)
    for k, v in change.items():
        setattr(d, k, v)
    names = ("x", "residual", "post_weight", "gate", "weight", "residual_out", "y", "scales")
    a = dict(zip(names, AT))
    a["scales"] = None
    a.update(at or {})
    a.update({n: None for n in null})
    return mf.lib.mafat_block_norm(ctypes.byref(d), *[a[n] for n in names], None)


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), "EINVAL"), (dict(dtype=2), "EINVAL"), (dict(out_dtype=1), "EINVAL"), (dict(cols=0), "EINVAL"),
    (dict(cols=16385), "EUNSUPPORTED"), (dict(rows=-1), "EINVAL"), (dict(rows=1 << 31), "EUNSUPPORTED"),
    (dict(rows=(1 << 31) - 1, x_stride=1 << 39), "EUNSUPPORTED"), (dict(rows=(1 << 31) - 1, gate_rows=1, gate_stride=1 << 32), "EUNSUPPORTED"),
    (dict(eps=-1.0), "EINVAL"),
    (dict(eps=math.nan), "EINVAL"), (dict(eps=math.inf), "EINVAL"), (dict(branch_scale=math.inf), "EINVAL"),
    (dict(residual_scale=math.nan), "EINVAL"), (dict(scale_group=128), "EINVAL"), (dict(gate_rows=-1), "EINVAL"),
    (dict(gate_rows=5), "EINVAL"), (dict(gate_rows=24), "EINVAL"), (dict(x_stride=255), "EINVAL"), (dict(gate_stride=-256), "EINVAL"),
    (dict(y_stride=1 << 41), "EUNSUPPORTED"), (dict(out_dtype=2), "EINVAL"), (dict(null=("x",)), "EINVAL"),
    (dict(null=("residual",)), "EINVAL"), (dict(null=("y",)), "EINVAL"), (dict(null=("weight",)), "EINVAL"),
    (dict(null=("weight", "y", "residual_out")), "EINVAL"), (dict(at=dict(scales=4096)), "EINVAL"),
    (dict(at=dict(gate=AT[3] + 8)), "EINVAL"), (dict(at=dict(y=AT[2])), "EINVAL"), (dict(at=dict(y=AT[3])), "EINVAL"),
    (dict(at=dict(residual_out=AT[4])), "EINVAL"), (dict(at=dict(residual_out=AT[6])), "EINVAL"),
    (dict(at=dict(residual_out=AT[0] + 16)), "EINVAL"), (dict(at=dict(y=AT[0]), x_stride=512), "EINVAL"),
    (dict(out_dtype=2, at=dict(scales=4096, y=AT[0])), "EINVAL"), (dict(out_dtype=2, at=dict(scales=4098)), "EINVAL"),
    (dict(out_dtype=2, scale_group=64, at=dict(scales=4096)), "EUNSUPPORTED"), (dict(out_dtype=2, null=("weight", "y"), at=dict(scales=4096)), "EINVAL")])
def test_norm_refusals(mf, change, status):
    _status(mf, _norm(mf, **change), status)


def test_norm_of_no_rows(mf):
    assert _norm(mf, rows=0, null=("x", "y", "residual")) == mf.OK
    assert mf.lib.mafat_block_norm(None, *[None] * 9) == mf.EINVAL


# ---- rotary positions ---------------------------------------------------------------------------


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=0), "EINVAL"), (dict(head_dim=12), "EUNSUPPORTED"), (dict(head_dim=264), "EUNSUPPORTED"), (dict(rot_dim=3), "EINVAL"),
    (dict(rot_dim=66), "EINVAL"), (dict(rot_dim=-2), "EINVAL"), (dict(dtype=2), "EINVAL"), (dict(scaling=4), "EINVAL"),
    (dict(scaling=-1), "EINVAL"), (dict(base=1.0), "EINVAL"), (dict(base=math.inf), "EINVAL"), (dict(base=math.nan), "EINVAL"),
    (dict(factor=2.0), "EINVAL"), (dict(scaling=1, factor=0.5), "EINVAL"), (dict(scaling=1, factor=math.nan), "EINVAL"),
    (dict(scaling=2, rot_dim=2, factor=2.0), "EINVAL"), (dict(scaling=3, factor=2.0), "EINVAL"),
    (dict(scaling=3, factor=2.0, first_positions=100, fast=1.0, slow=1.0), "EINVAL"),
    (dict(scaling=3, factor=2.0, first_positions=100, fast=2.0), "EINVAL"), (dict(magnitude=-1.0), "EINVAL"),
    (dict(magnitude=math.inf), "EINVAL"), (dict(frequencies=[1.0] * 31), "EINVAL"), (dict(frequencies=[math.nan] * 32), "EINVAL"),
    (dict(frequencies=[65537.0] * 32), "EINVAL"), (dict(frequencies=[1.0] * 32, base=100.0), "EINVAL"),
    (dict(frequencies=[1.0] * 32, scaling=1), "EINVAL")])
def test_rotary_plans(mf, change, status):
    with pytest.raises(mf.MafatError) as e:
        mf.Rotary(**{**dict(head_dim=64, dry_run=True), **change})
    assert mf.STATUS[e.value.status] == status, str(e.value)


def _rotary(mf, at=None, null=(), plan=None, **change):
    plan = plan or mf.Rotary(64, dry_run=True)
    c = mf.RotaryCall(struct_size=ctypes.sizeof(mf.RotaryCall), batch=2, n_q=3, heads_q=4, heads_kv=2, room=10)
    for k, v in change.items():
        if isinstance(v, tuple):
            getattr(c, k)[:] = v
        else:
            setattr(c, k, v)
    names = ("positions", "places", "q", "q_out", "k", "k_out", "v", "v_out")
    a = dict(zip(names, AT))
    a.update(at or {})
    a.update({n: None for n in null})
    return mf.lib.mafat_rotary_run(plan.handle, ctypes.byref(c), *[a[n] for n in names], None)


SIDE = (3 * 512, 512, 64)  # of a matrix whose rows are 4 queries, 2 keys, 2 values


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=1), "EINVAL"), (dict(batch=-1), "EINVAL"), (dict(n_q=-1), "EINVAL"), (dict(heads_q=0), "EINVAL"),
    (dict(heads_kv=0), "EINVAL"), (dict(heads_kv=-2), "EINVAL"), (dict(room=-1), "EINVAL"), (dict(heads_q=1 << 20), "EUNSUPPORTED"),
    (dict(batch=1 << 20, n_q=1 << 20), "EUNSUPPORTED"), (dict(null=("places",)), "EINVAL"), (dict(null=("positions",)), "EINVAL"),
    (dict(null=("q",)), "EINVAL"), (dict(null=("k_out",)), "EINVAL"), (dict(null=("q", "q_out", "k", "k_out", "v", "v_out")), "EINVAL"),
    (dict(at=dict(positions=AT[0] + 2)), "EINVAL"), (dict(at=dict(k=AT[4] + 8)), "EINVAL"), (dict(q_strides=(768, 256, 60)), "EINVAL"),
    (dict(q_out_strides=(768, 256, 68)), "EINVAL"), (dict(k_out_strides=(128, 128, 64)), "EINVAL"), (dict(q_strides=(1 << 41, 256, 64)), "EUNSUPPORTED"),
    (dict(at=dict(q_out=AT[4])), "EINVAL"), (dict(at=dict(k_out=AT[4])), "EINVAL"), (dict(at=dict(v_out=AT[5])), "EINVAL"),
    (dict(at=dict(q_out=AT[2] + 16)), "EINVAL"), (dict(at=dict(q_out=AT[2]), q_strides=SIDE), "EINVAL"),
    (dict(at=dict(k_out=AT[0])), "EINVAL"),
    # keys that reach into the queries' heads, and into the next row's
    (dict(at=dict(q_out=AT[2], k=AT[2] + 192 * 2), q_strides=SIDE, q_out_strides=SIDE, k_strides=SIDE), "EINVAL"),
    (dict(at=dict(q_out=AT[2], k=AT[2] + 448 * 2), q_strides=SIDE, q_out_strides=SIDE, k_strides=SIDE), "EINVAL"),
    (dict(at=dict(q_out=AT[2], k=AT[2] + 256 * 2), q_strides=SIDE, q_out_strides=SIDE, k_strides=(3 * 512, 520, 64)), "EINVAL")])
def test_rotary_runs(mf, change, status):
    _status(mf, _rotary(mf, **change), status)


def test_rotary_calls_that_reach_the_launch(mf):
    """What is not refused comes to the plan's being a dry run."""
    for change in (dict(), dict(null=("places",), room=3), dict(null=("q", "q_out")), dict(null=("k", "k_out", "v", "v_out")),
                   dict(at=dict(q_out=AT[2], k=AT[2] + 256 * 2, v=AT[2] + 384 * 2), q_strides=SIDE, q_out_strides=SIDE, k_strides=SIDE, v_strides=SIDE),
                   dict(at=dict(q_out=AT[2], k=AT[2] + 256 * 2, k_out=AT[2] + 256 * 2), null=("places",), room=3, q_strides=SIDE, q_out_strides=SIDE,
                        k_strides=SIDE, k_out_strides=SIDE)):
        assert _rotary(mf, **change) == mf.EINVAL and b"dry_run" in mf.lib.mafat_last_error()
    assert _rotary(mf, batch=0, null=("q", "positions")) == mf.OK and _rotary(mf, n_q=0, null=("positions",)) == mf.OK
    assert _rotary(mf, room=0, null=("q", "q_out", "k_out", "v_out")) == mf.OK
    h = ctypes.c_void_p()
    assert mf.lib.mafat_rotary_plan(None, ctypes.byref(h)) == mf.EINVAL
    assert mf.lib.mafat_rotary_plan(ctypes.byref(mf.RotaryDesc()), ctypes.byref(h)) == mf.EINVAL
    assert mf.lib.mafat_rotary_plan(ctypes.byref(mf.RotaryDesc()), None) == mf.EINVAL
    assert mf.lib.mafat_rotary_run(None, None, *[None] * 9) == mf.EINVAL
    assert mf.lib.mafat_rotary_frequencies(None, None, None) == mf.EINVAL
    mf.lib.mafat_rotary_destroy(None)


# ---- trees ----------------------------------------------------------------------------------------


TREE = dict(prefixes=2, requests=3, n_q=5, n_prefix=100, n_own=20, heads_q=8, heads_kv=2, head_dim=64, dry_run=True)


@pytest.mark.parametrize("change,status", [
    (dict(prefixes=0), "EINVAL"), (dict(requests=0), "EINVAL"), (dict(n_prefix=-1), "EINVAL"), (dict(n_own=-5), "EINVAL"),
    (dict(n_q=0), "EINVAL"), (dict(heads_q=7), "EINVAL"), (dict(head_dim=20), "EUNSUPPORTED"), (dict(own_k_strides=(2560, 64, 60)), "EINVAL"),
    (dict(prefixes=1 << 20, requests=1 << 20), "EUNSUPPORTED"), (dict(out_strides=(512, 512, 64)), "EINVAL")])
def test_tree_plans(mf, change, status):
    with pytest.raises(mf.MafatError) as e:
        mf.TreeAttention(**{**TREE, **change})
    assert mf.STATUS[e.value.status] == status, str(e.value)


def test_kinds_of_plans_are_told_apart(mf):
    tree, prefix = mf.TreeAttention(**TREE), mf.PrefixAttention(**TREE)
    assert mf.lib.mafat_prefix_run(tree.handle, *[4096] * 11) == mf.EINVAL and b"mafat_tree_plan" in mf.lib.mafat_last_error()
    assert mf.lib.mafat_cross_run(tree.handle, *[4096] * 8) == mf.EINVAL and b"mafat_tree_plan" in mf.lib.mafat_last_error()
    assert mf.lib.mafat_tree_run(prefix.handle, *[4096] * 10, 0, *[4096] * 3) == mf.EINVAL
    assert b"mafat_prefix_plan" in mf.lib.mafat_last_error()
    assert mf.lib.mafat_tree_run(tree.handle, *[4096] * 10, 0, *[4096] * 3) == mf.EINVAL and b"dry_run" in mf.lib.mafat_last_error()
    assert mf.lib.mafat_tree_run(None, *[4096] * 10, 0, *[4096] * 3) == mf.EINVAL
    assert mf.lib.mafat_tree_plan(None, ctypes.byref(ctypes.c_void_p())) == mf.EINVAL
    assert mf.lib.mafat_tree_plan(ctypes.byref(mf.PrefixDesc()), ctypes.byref(ctypes.c_void_p())) == mf.EINVAL


# ---- logits ---------------------------------------------------------------------------------------


LOGITS = ("logits", "tokens", "lengths", "prompt_lengths", "repetition", "presence", "frequency", "drafts", "tree", "bias_ids", "bias",
          "masks", "mask_rows", "out")


def _logits(mf, at=None, null=(), **change):
    d = mf.LogitsDesc(struct_size=ctypes.sizeof(mf.LogitsDesc), dtype=1, out_dtype=1, batch=2, n_q=3, vocab=1000, room=50, n_bias=4, n_masks=5)
    for k, v in change.items():
        setattr(d, k, v)
    a = dict(zip(LOGITS, AT))
    a.update(at or {})
    a.update({n: None for n in null})
    return mf.lib.mafat_adjust_logits(ctypes.byref(d), *[a[n] for n in LOGITS], None)


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=1), "EINVAL"), (dict(dtype=2), "EINVAL"), (dict(out_dtype=0), "EINVAL"), (dict(batch=-1), "EINVAL"), (dict(n_q=-1), "EINVAL"),
    (dict(vocab=0), "EINVAL"), (dict(vocab=(1 << 30) + 1), "EUNSUPPORTED"),
    (dict(batch=1 << 30, n_q=(1 << 18) - 64, vocab=1 << 30), "EUNSUPPORTED"), (dict(room=-1), "EINVAL"), (dict(room=(1 << 18) - 3), "EUNSUPPORTED"),
    (dict(n_bias=-1), "EINVAL"), (dict(n_bias=4096), "EUNSUPPORTED"), (dict(n_masks=-1), "EINVAL"), (dict(batch=1 << 30), "EUNSUPPORTED"),
    (dict(logits_stride=999), "EINVAL"), (dict(out_stride=-1000), "EINVAL"), (dict(out_stride=1 << 31), "EUNSUPPORTED"),
    (dict(null=("logits",)), "EINVAL"), (dict(null=("out",)), "EINVAL"), (dict(null=("bias",)), "EINVAL"), (dict(null=("bias_ids",)), "EINVAL"),
    (dict(null=("drafts",)), "EINVAL"), (dict(null=("masks",)), "EINVAL"), (dict(null=("mask_rows",)), "EINVAL"), (dict(null=("tokens",)), "EINVAL"),
    (dict(at=dict(logits=AT[0] + 2)), "EINVAL"), (dict(at=dict(tree=AT[8] + 2)), "EINVAL"), (dict(at=dict(out=AT[0] + 4)), "EINVAL"),
    (dict(at=dict(out=AT[0]), out_stride=1001), "EINVAL"), (dict(at=dict(out=AT[0]), dtype=0), "EINVAL")]
    + [(dict(at=dict(out=a)), "EINVAL") for a in AT[1:13]])
def test_logits_refusals(mf, change, status):
    _status(mf, _logits(mf, **change), status)


def test_logits_of_no_rows(mf):
    assert _logits(mf, batch=0, null=LOGITS) == mf.OK and _logits(mf, n_q=0, null=LOGITS) == mf.OK
    assert mf.lib.mafat_adjust_logits(None, *[None] * 15) == mf.EINVAL


# ---- tensors, before the library sees their addresses ---------------------------------------------


class OnGpu:
    """A host tensor that says it is on GPU `device`."""
    is_cuda = True

    def __init__(self, t, device=0):
        self.t, self.index = t, device

    def get_device(self):
        return self.index

    @property
    def device(self):
        return torch.device("cuda", self.index)

    def __getitem__(self, i):
        return OnGpu(self.t[i], self.index)

    def __getattr__(self, name):
        return getattr(self.t, name)


def _calls(mf):
    """For each operator: its entry point, the call, its tensors."""
    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)

    def ints(*shape):
        return torch.zeros(shape, dtype=torch.int32)
    rotary, tree = mf.Rotary(64, dry_run=True), mf.TreeAttention(2, 2, 5, 30, 10, 4, 2, 64, dry_run=True)
    return {
        "norm": ("mafat_block_norm", lambda **k: mf.block_norm(stream=0, **k), dict(
            x=bf16(6, 64), residual=bf16(6, 64), residual_out=bf16(6, 64), post_weight=bf16(64), gate=bf16(3, 64), weight=bf16(64),
            y=torch.zeros(6, 64).to(torch.float8_e4m3fn), scales=torch.zeros(6, 1))),
        "rotary": ("mafat_rotary_run", lambda **k: rotary.run(stream=0, **k), dict(
            positions=ints(2, 3), q=bf16(2, 3, 4, 64), q_out=bf16(2, 3, 4, 64), k=bf16(2, 3, 2, 64), k_out=bf16(2, 9, 2, 64),
            v=bf16(2, 3, 2, 64), v_out=bf16(2, 9, 2, 64), places=ints(2, 3))),
        "tree": ("mafat_tree_run", lambda **k: tree.run(stream=0, **k), dict(
            q=bf16(4, 5, 4, 64), prefix_k=bf16(2, 30, 2, 64), prefix_v=bf16(2, 30, 2, 64), own_k=bf16(4, 10, 2, 64), own_v=bf16(4, 10, 2, 64),
            tree=ints(4, 5, 1), out=bf16(4, 5, 4, 64), nodes=ints(4), prefix_len=ints(2), prefix_mask=torch.ones(2, 30, dtype=torch.bool),
            own_len=ints(4), lse=torch.zeros(4, 5, 4))),
        "logits": ("mafat_adjust_logits", lambda **k: mf.adjust_logits(stream=0, **k), dict(
            logits=bf16(2, 3, 100), out=torch.zeros(2, 3, 100), tokens=ints(2, 20), lengths=ints(2), prompt_lengths=ints(2),
            repetition=torch.ones(2), presence=torch.ones(2), frequency=torch.ones(2), drafts=ints(2, 3), tree=ints(2, 3, 1),
            bias_ids=ints(2, 4), bias=torch.zeros(2, 4), masks=ints(5, 4), mask_rows=ints(2, 3))),
    }


@pytest.mark.parametrize("which", ["norm", "rotary", "tree", "logits"])
def test_tensors_that_are_refused(mf, monkeypatch, which):
    """Of another GPU or the host, of another type or size, spread channels, rows that are shared."""
    monkeypatch.setattr(mf, "_current_device", lambda: 0)
    entry, call, tensors = _calls(mf)[which]
    seen = []
    monkeypatch.setattr(mf.lib, entry, lambda *a: seen.append(a) or mf.OK)
    here = {n: OnGpu(t) for n, t in tensors.items()}
    call(**here)
    assert len(seen) == 1
    for name, t in tensors.items():
        wrong = [OnGpu(t, 1), t, OnGpu(t.to(torch.float64))] + ([OnGpu(torch.cat([t, t], -1))] if name != "tokens" else [])
        if t.dim() > 1:
            wide = torch.zeros(t.shape[:-1] + (2 * t.shape[-1],)).to(t.dtype)
            wrong.append(OnGpu(wide[..., ::2]) if t.shape[-1] > 1 else OnGpu(torch.cat([t, t], 0)))
            wrong.append(OnGpu(t[:1].expand(t.shape)))
        for w in wrong:
            if (which, name) in (("logits", "out"), ("logits", "logits"), ("norm", "y")) and w.dtype == torch.float64:
                continue  # the library's to refuse
            with pytest.raises(mf.MafatError) as e:
                call(**{**here, name: w})
            assert e.value.status == mf.EINVAL, name
    assert len(seen) == 1


def test_forms_that_are_taken(mf, monkeypatch):
    monkeypatch.setattr(mf, "_current_device", lambda: 0)
    calls = _calls(mf)
    seen = []
    for entry in ("mafat_block_norm", "mafat_rotary_run", "mafat_tree_run", "mafat_adjust_logits"):
        monkeypatch.setattr(mf.lib, entry, lambda *a: seen.append(a) or mf.OK)
    norm, rotary, tree, logits = ({n: OnGpu(t) for n, t in calls[k][2].items()} for k in ("norm", "rotary", "tree", "logits"))
    calls["norm"][1](**{**norm, "gate": OnGpu(torch.zeros(64, dtype=torch.bfloat16))})
    assert seen[-1][0].gate_rows == 6
    calls["norm"][1](**{**norm, "gate": OnGpu(torch.zeros(3, 80, dtype=torch.bfloat16)[:, :64])})
    assert seen[-1][0].gate_rows == 2 and seen[-1][0].gate_stride == 80
    side = torch.zeros(2, 3, 8, 64, dtype=torch.bfloat16)
    calls["rotary"][1](**{**rotary, "q": OnGpu(side[:, :, :4]), "k": OnGpu(side[:, :, 4:6])})
    assert list(seen[-1][1].q_strides) == [1536, 512, 64] and seen[-1][1].room == 9
    calls["tree"][1](**{**tree, "tree": OnGpu(torch.zeros(1, 5, 1, dtype=torch.int32))})
    assert seen[-1][11] == 1
    calls["tree"][1](**tree)
    assert seen[-1][11] == 0
    calls["logits"][1](**{**logits, "tree": OnGpu(torch.zeros(1, 3, 1, dtype=torch.int32)), "bias_ids": OnGpu(torch.zeros(1, 4, dtype=torch.int32)),
                          "bias": OnGpu(torch.zeros(1, 4))})
    assert seen[-1][0].tree_shared == 1 and seen[-1][0].bias_shared == 1
    wide = torch.zeros(2, 3, 128, dtype=torch.bfloat16)[..., :100]
    calls["logits"][1](**{**logits, "logits": OnGpu(wide)})
    assert seen[-1][0].logits_stride == 128 and seen[-1][0].out_stride == 100
    with pytest.raises(mf.MafatError):  # rows that are not apart by one step
        calls["logits"][1](**{**logits, "logits": OnGpu(torch.zeros(2, 4, 100, dtype=torch.bfloat16)[:, :3])})
    two = {n: logits[n] for n in ("tokens", "lengths", "repetition")}
    mf.adjust_logits(OnGpu(torch.zeros(2, 100)), OnGpu(torch.zeros(2, 100)), masks=OnGpu(torch.zeros(5, 4, dtype=torch.int32)),
                     mask_rows=OnGpu(torch.zeros(2, dtype=torch.int32)), stream=0, **two)
    assert seen[-1][0].n_q == 1


def test_calls_that_are_kept_are_told_apart(mf, monkeypatch):
    """More kinds of calls than are kept, in turn: each reaches the library with its own sizes, strides and addresses."""
    monkeypatch.setattr(mf, "_current_device", lambda: 0)
    seen = []
    for entry in ("mafat_block_norm", "mafat_adjust_logits", "mafat_rotary_run"):
        monkeypatch.setattr(mf.lib, entry, lambda *a: seen.append(a) or mf.OK)
    rotary = mf.Rotary(64, dry_run=True)
    rotary.device = 0
    kinds = [(rows, cols, pad) for rows in (2, 3, 5) for cols in (64, 72, 96) for pad in (0, 8)]
    assert len(kinds) > mf.MOST_CALLS
    for turn in range(3):
        for rows, cols, pad in kinds:
            x, r, h = (OnGpu(torch.zeros(rows, cols + pad)[:, :cols]) for _ in range(3))
            for scale in (1.0, 0.5):
                mf.block_norm(x, r, h, branch_scale=scale, stream=0)
                d = seen[-1][0]
                assert (d.rows, d.cols, d.branch_scale) == (rows, cols, scale) and d.x_stride == cols + pad
                assert list(seen[-1][1:3]) == [x.data_ptr(), r.data_ptr()] and seen[-1][6] == h.data_ptr() and seen[-1][4] is None
            out = OnGpu(torch.zeros(rows, cols))
            tokens = OnGpu(torch.zeros(rows, 1 + turn, dtype=torch.int32))
            mf.adjust_logits(x, out, tokens=tokens, stream=0)
            d = seen[-1][0]
            assert (d.batch, d.vocab, d.room, d.logits_stride, d.out_stride) == (rows, cols, 1 + turn, cols + pad, cols)
            assert seen[-1][1] == x.data_ptr() and seen[-1][2] == tokens.data_ptr() and seen[-1][-2] == out.data_ptr()
            q = OnGpu(torch.zeros(rows, 2, cols // 8, 64 + pad, dtype=torch.bfloat16)[..., :64])
            o = OnGpu(torch.zeros(rows, 2, cols // 8, 64, dtype=torch.bfloat16))
            at = OnGpu(torch.zeros(rows, 2, dtype=torch.int32))
            rotary.run(at, q=q, q_out=o, stream=0)
            d = seen[-1][1]
            assert (d.batch, d.heads_q, d.q_strides[2]) == (rows, cols // 8, 64 + pad) and seen[-1][4:6] == (q.data_ptr(), o.data_ptr())
    assert len(mf._norm_calls) <= mf.MOST_CALLS and len(rotary._calls) <= mf.MOST_CALLS


def test_what_is_not_a_tensor(mf, monkeypatch):
    """Raw addresses are the caller's word where shapes are not asked for; anything else is an error, not a match."""
    plan = mf.TreeAttention(2, 2, 5, 30, 10, 4, 2, 64, dry_run=True)
    seen = []
    monkeypatch.setattr(mf.lib, "mafat_tree_run", lambda *a: seen.append(a) or mf.OK)
    plan.device = 0
    plan._types = mf._type(mf.BF16), mf._type("int32"), mf._type("mask"), mf._type(mf.FP32)
    for _ in range(2):
        plan.run(*[4096 * (i + 1) for i in range(7)], stream=0)
    assert len(seen) == 2 and not plan._calls and seen[0][1] == 4096


def test_calls_made_by_the_module(mf, monkeypatch):
    """Calls that are like one made before go to the library itself, whose refusals of made-up addresses come back; the rest
    is as if they were the first."""
    monkeypatch.setattr(mf, "_current_device", lambda: 0)
    entry, call, tensors = _calls(mf)["norm"]
    seen = []
    real = mf.lib.mafat_block_norm
    monkeypatch.setattr(mf, "_norm_calls", [])
    monkeypatch.setattr(mf.lib, entry, lambda *a: seen.append(a) or mf.OK)
    here = {n: OnGpu(t) for n, t in tensors.items()}
    call(**here)
    assert len(seen) == 1 and len(mf._norm_calls) == 1
    here["residual_out"] = here["gate"]  # of another shape: not like it, and refused
    with pytest.raises(mf.MafatError):
        call(**here)
    whole = torch.zeros(6 * 64 + 8, dtype=torch.bfloat16)
    for shift in (8, 16):  # outputs that overlap an input, or are not aligned: the library's word
        x = OnGpu(whole[:384].view(6, 64))
        at = whole[shift:shift + 384] if shift == 8 else whole[4:388]
        with pytest.raises(mf.MafatError) as e:
            call(**{**here, "x": x, "residual_out": OnGpu(at.view(6, 64))})
        assert e.value.status == mf.EINVAL and ("overlaps" in str(e.value) or "aligned" in str(e.value))
    assert len(seen) == 1 and real is not mf.lib.mafat_block_norm


def test_the_module_checks_its_arguments(mf):
    run = mf._match.run
    for args in ((0, [], [], 0, None, None, None), (0, (), (), 0, None, None, None), ("0", [], (), 0, None, None, None), (0, [])):
        with pytest.raises(TypeError):
            run(*args)
    for args in ((4, [], (), 0, None, None, None), (-1, [], (), 0, None, None, None), (0, [], (None,) * 7, 0, None, None, None)):
        with pytest.raises(ValueError):
            run(*args)
    none = (None,) * 8
    assert run(0, [], none, 0, None, None, None) is None
    assert run(0, [(none, 1, 0)], none, 0, 2, None, None) is None and run(0, [(none[1:], 1, 0)], none, 0, 1, None, None) is None
    look = (torch.float32, (2,), None)
    assert run(0, [((look,) + none[1:], 1, 0)], (object(),) + none[1:], 0, 1, None, None) is None
    assert run(0, [(none, 1, 0)], none, 0, 1, None, None) == mf.EINVAL  # a null descriptor, by the library


@pytest.mark.parametrize("which", ["norm", "rotary", "tree", "logits"])
def test_refused_calls_are_not_kept(mf, monkeypatch, which):
    """Those that the library refuses leave the kept ones as they were."""
    monkeypatch.setattr(mf, "_current_device", lambda: 0)
    monkeypatch.setattr(mf, "_norm_calls", [])
    monkeypatch.setattr(mf, "_logits_calls", [])
    entry, call, tensors = _calls(mf)[which]
    if which in ("rotary", "tree"):
        plan = [c.cell_contents for c in call.__closure__][0]
        plan.device = 0
    calls = {"norm": lambda: mf._norm_calls, "logits": lambda: mf._logits_calls}.get(which, lambda: plan._calls)
    here = {n: OnGpu(t) for n, t in tensors.items()}
    with monkeypatch.context() as m:
        m.setattr(mf.lib, entry, lambda *a: mf.EINVAL)
        for _ in range(2):
            with pytest.raises(mf.MafatError):
                call(**here)
            assert calls() == []
        m.setattr(mf.lib, entry, lambda *a: mf.OK)
        call(**here)
        kept = list(calls())
        m.setattr(mf.lib, entry, lambda *a: mf.EUNSUPPORTED)
        fewer = {"norm": "gate", "rotary": "places", "tree": "lse", "logits": "masks"}[which]
        more = {"rotary": dict(k_out=here.get("k"), v_out=here.get("v")), "logits": dict(mask_rows=None)}.get(which, {})
        with pytest.raises(mf.MafatError) as e:
            call(**{**here, fewer: None, **more})
        assert e.value.status == mf.EUNSUPPORTED and len(kept) == 1 and list(calls()) == kept


@pytest.mark.parametrize("null,sizes", [
    (("tokens",), dict(room=0)), (("tokens", "lengths"), dict(room=0)), (("tokens", "prompt_lengths"), dict(room=0)),
    (("masks",), dict(n_masks=0)), (("tokens", "masks", "bias_ids", "bias"), dict(room=0, n_masks=0, n_bias=0))])
def test_lists_of_nothing(mf, null, sizes):
    """A tensor without elements has no address: what goes with it is taken, and the call refused for its output alone."""
    assert _logits(mf, null=null, at=dict(out=AT[0]), out_stride=1001, **sizes) == mf.EINVAL
    assert mf.lib.mafat_last_error() == b"an output overlaps another tensor"


@pytest.mark.parametrize("which", ["rotary", "tree"])
def test_closed_plans(mf, monkeypatch, which):
    entry, call, tensors = _calls(mf)[which]
    plan = [c.cell_contents for c in call.__closure__][0]
    plan.device = 0  # as of a plan for the GPU: its calls are kept
    here = {n: OnGpu(t) for n, t in tensors.items()}
    with monkeypatch.context() as m:
        m.setattr(mf.lib, entry, lambda *a: mf.OK)
        call(**here)
    assert len(plan._calls) == 1
    plan.close()
    for _ in range(2):
        with pytest.raises(mf.MafatError) as e:
            call(**here)
        assert e.value.status == mf.EINVAL
