"""What the language operators say to tensors before the library sees their addresses.  The tensors are stand-ins that
say they are on a GPU; a recorder stands in for the library's entry points, so that nothing is launched."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


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

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture()
def norm_calls(mf, monkeypatch):
    """The descriptors that reach mafat_rms_norm."""
    calls = []

    def record(desc, *addresses):
        calls.append(desc._obj)
        return mf.OK
    monkeypatch.setattr(mf.lib, "mafat_rms_norm", record)
    monkeypatch.setattr(mf, "_current_device", lambda: 0)
    return calls


def _rows(rows=16, cols=256, **kw):
    return OnGpu(torch.ones(rows, cols), **kw)


def _weight(cols=256, **kw):
    return OnGpu(torch.ones(cols), **kw)


@pytest.mark.parametrize("which", ["x", "residual", "residual_out", "y"])
@pytest.mark.parametrize("cols", [1, 256])
def test_broadcast_rows_are_refused(mf, norm_calls, which, cols):
    """A row expanded to many has a stride of 0, which stands for packed rows in the descriptor."""
    tensors = {n: _rows(cols=cols) for n in ("x", "residual", "residual_out", "y")}
    mf.rms_norm(weight=_weight(cols), stream=0, **tensors)
    assert len(norm_calls) == 1
    tensors[which] = OnGpu(torch.ones(1, cols).expand(16, cols))
    with pytest.raises(mf.MafatError) as e:
        mf.rms_norm(weight=_weight(cols), stream=0, **tensors)
    assert e.value.status == mf.EINVAL and which in str(e.value)
    assert len(norm_calls) == 1


@pytest.mark.parametrize("which", ["x", "residual", "residual_out", "y"])
def test_strides_of_rows_reach_the_library(mf, norm_calls, which):
    """Rows of a wider matrix, and a single row, whose stride is nothing to go by."""
    fields = {"x": "x_stride", "residual": "residual_stride", "residual_out": "residual_out_stride", "y": "y_stride"}
    tensors = {n: _rows() for n in fields}
    tensors[which] = OnGpu(torch.ones(16, 300)[:, :256])
    mf.rms_norm(weight=_weight(), stream=0, **tensors)
    assert [getattr(norm_calls[-1], f) for f in fields.values()] == [300 if n == which else 256 for n in fields]
    tensors = {n: _rows(1) for n in fields}
    tensors[which] = OnGpu(torch.as_strided(torch.ones(256), (1, 256), (0, 1)))
    mf.rms_norm(weight=_weight(), stream=0, **tensors)
    assert all(getattr(norm_calls[-1], f) in (0, 256) for f in fields.values())


# ---- tensors on another GPU than the current one -----------------------------------------------


@pytest.fixture()
def on_gpu_0(mf, monkeypatch):
    monkeypatch.setattr(mf, "_current_device", lambda: 0)


@pytest.mark.parametrize("packed", [True, False])
def test_norms_of_another_gpu_are_refused(mf, norm_calls, on_gpu_0, packed):
    def make(device=0):
        e4m3 = torch.zeros(16, 256).to(torch.float8_e4m3fn)
        rows = {n: torch.ones(16, 256) if packed else torch.ones(16, 300)[:, :256] for n in ("x", "residual", "residual_out")}
        return {n: OnGpu(t, device) for n, t in dict(weight=torch.ones(256), y=e4m3, scales=torch.ones(16, 1), **rows).items()}
    here, there = make(), make(1)
    mf.rms_norm(stream=0, **here)
    assert len(norm_calls) == 1
    for name in here:
        with pytest.raises(mf.MafatError) as e:
            mf.rms_norm(stream=0, **{**here, name: there[name]})
        assert e.value.status == mf.EINVAL, name
    with pytest.raises(mf.MafatError) as e:  # all of one GPU, which is not the one that kernels are launched on
        mf.rms_norm(stream=0, **there)
    assert e.value.status == mf.EINVAL and "cuda:1" in str(e.value)
    with pytest.raises(mf.MafatError):
        mf.rms_norm(stream=0, **{**here, "x": torch.ones(16, 256)})  # of the host
    with pytest.raises(mf.MafatError):
        mf.rms_norm(stream=0, **{n: t.t for n, t in here.items()})
    assert len(norm_calls) == 1


def _attention(mf, kind):
    """A plan and what its run takes."""
    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)
    q = bf16(4, 1, 4, 64)
    if kind == "cross":
        return mf.CrossAttention(4, 1, 30, 4, 2, 64, dry_run=True), dict(
            q=q, k=bf16(4, 30, 2, 64), v=bf16(4, 30, 2, 64), out=q.clone(), kv_len=torch.zeros(4, dtype=torch.int32),
            kv_mask=torch.ones(4, 30, dtype=torch.uint8), lse=torch.zeros(4, 1, 4))
    return mf.PrefixAttention(2, 2, 1, 30, 10, 4, 2, 64, dry_run=True), dict(
        q=q, prefix_k=bf16(2, 30, 2, 64), prefix_v=bf16(2, 30, 2, 64), own_k=bf16(4, 10, 2, 64), own_v=bf16(4, 10, 2, 64),
        out=q.clone(), prefix_len=torch.zeros(2, dtype=torch.int32), prefix_mask=torch.ones(2, 30, dtype=torch.bool),
        own_len=torch.zeros(4, dtype=torch.int32), lse=torch.zeros(4, 1, 4))


@pytest.mark.parametrize("kind", ["cross", "prefix"])
def test_attention_of_another_gpu_is_refused(mf, monkeypatch, on_gpu_0, kind):
    plan, tensors = _attention(mf, kind)
    calls = []
    monkeypatch.setattr(mf.lib, "mafat_%s_run" % kind, lambda *a: calls.append(a) or mf.OK)
    here = {n: OnGpu(t) for n, t in tensors.items()}
    plan.run(stream=0, **here)
    plan.run(stream=0, **{**here, "q": 4096})  # an address is the caller's word
    plan.run(stream=0, **{n: 4096 for n in here})
    assert len(calls) == 3
    for name in tensors:
        with pytest.raises(mf.MafatError) as e:
            plan.run(stream=0, **{**here, name: OnGpu(tensors[name], 1)})
        assert e.value.status == mf.EINVAL, name
        with pytest.raises(mf.MafatError):
            plan.run(stream=0, **{**here, name: tensors[name]})
    with pytest.raises(mf.MafatError) as e:
        plan.run(stream=0, **{n: OnGpu(t, 1) for n, t in tensors.items()})
    assert e.value.status == mf.EINVAL and "cuda:1" in str(e.value)
    with pytest.raises(mf.MafatError):
        plan.run(stream=0, **tensors)
    assert len(calls) == 3
