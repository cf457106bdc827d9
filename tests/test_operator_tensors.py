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
