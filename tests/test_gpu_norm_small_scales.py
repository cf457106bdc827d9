"""8-bit norms so small that a scale has few bits, or none."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("rows", [5, 2100])
@pytest.mark.parametrize("cols", [512, 330, 251])
@pytest.mark.parametrize("size", [2e-44, 1e-43, 5e-42, 1e-38])
def test_small_norms(mf, dt, group, rows, cols, size):
    """Norms of `size`, some of them zero.  A block whose largest norm / 448 is zero in fp32 has scale 1, as one of zeros
    has; its values are below 448 * 2^-150 and become 0.  Else a scale is a multiple of 2^-149, off by 2^-150 at most, and so
    is the norm: 450 of these bound what the two take away (448 of them where the quotient saturates), next to half a step of
    8 bits: 2^-4 of a value, 2^-10 of the scale."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + cols)
    # the squares vanish beside eps, whose root is a power of two: norms are x * 2^-30 * w
    x = (torch.randn((rows, cols), generator=g, device="cuda") * 2.0 ** -90).to(dt)
    x[:, ::7] = 0
    x[1, :128] = 0
    eps = 2.0 ** 60
    w = torch.full((cols,), size * 2.0 ** 120, device="cuda").to(dt)
    y = torch.full((rows, cols), 1.0, device="cuda").to(E4M3)
    n = -(-cols // 128) if group else 1
    s = torch.full((rows, n), -1.0, device="cuda")
    mf.rms_norm(x, w, y, scales=s, scale_group=group, eps=eps)
    ref = x.double() * 2.0 ** -30 * w.double()
    got = y.float().double()
    assert torch.isfinite(got).all() and torch.isfinite(s).all() and (s > 0).all()
    assert (got[x == 0] == 0).all()
    for i in range(n):
        c = slice(128 * i, 128 * (i + 1)) if group else slice(None)
        top = ref[:, c].abs().amax(-1)
        si = s[:, i].double()
        none, some = top < 448 * 2.0 ** -151, top > 448 * 2.0 ** -149  # between them rounding decides
        assert (si[none] == 1).all() and (got[:, c][none] == 0).all()
        assert ((si - top / 448).abs()[some] <= 2.0 ** -149 + 2.0 ** -20 * top[some] / 448).all()
        tol = 2.0 ** -4 * ref[:, c].abs() * (1 + 2.0 ** -18) + 2.0 ** -10 * si[:, None] + 450 * 2.0 ** -150
        assert ((got[:, c] * si[:, None] - ref[:, c]).abs()[some] <= tol[some]).all()
