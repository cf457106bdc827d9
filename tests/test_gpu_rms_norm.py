"""The root-mean-square norm against its definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _reference(x, r, w, eps):
    h = x.double() + (r.double() if r is not None else 0)
    return h, h / torch.sqrt(h.square().mean(-1, keepdim=True) + eps) * w.double()


def _tol32(cols):
    """h is rounded once before it is used (2^-24), the mean of squares is a sum of cols / 32 terms
    in a lane and of 32 * 16 at most after it ((cols / 32 + 16) 2^-24, half of it in the root), and
    root, division and two products add 2^-24 each."""
    return (cols / 32 + 32) * 2.0 ** -24


def _norm(mf, rows, cols, dt, quant=None, residual=True, pad=0, eps=1e-6, seed=1, change=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rows_of(fill=None, t=dt):
        b = torch.empty((rows, cols + pad), dtype=t, device="cuda")[:, :cols]
        return b if fill is None else b.copy_(fill)
    x = rows_of((torch.randn((rows, cols), generator=g, device="cuda") * 2))
    r = rows_of(torch.randn((rows, cols), generator=g, device="cuda")) if residual else None
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt)
    if change:
        change(x, r, w)
    h = rows_of() if residual else None
    y = rows_of(t=E4M3 if quant else dt)
    s = torch.empty((rows, 1 if quant == "row" else -(-cols // 128)), device="cuda") if quant else None
    mf.rms_norm(x, w, y, residual=r, residual_out=h, scales=s, scale_group=128 if quant == "128" else 0, eps=eps)
    h64, y64 = _reference(x, r, w, eps)
    out = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24  # half a step of 8 or 24 significant bits
    if residual:
        assert ((h.double() - h64).abs() <= (out + 2.0 ** -24) * h64.abs()).all()
    # h's own rounding in fp32 is relative to h, as are all others to y; a sum near zero of x and
    # r is exact in fp32 for bf16 inputs and rounded by 2^-24 of itself for fp32 ones
    t32 = _tol32(cols)
    if not quant:
        assert ((y.double() - y64).abs() <= (out + t32) * y64.abs() + 1e-37).all()
        return h, y, s
    width = cols if quant == "row" else 128
    for i in range(s.shape[1]):
        b = y64[:, i * width:(i + 1) * width]
        top = b.abs().amax(-1)
        want = torch.where(top == 0, torch.ones_like(top), top / 448)
        assert ((s[:, i].double() - want).abs() <= (t32 + 2.0 ** -23) * want).all()
        # 8 bits: half of 1/8 of the power of two below a value (2^-4 of it), or of the smallest step 2^-9
        q = b / want[:, None]
        got = y[:, i * width:(i + 1) * width].float().double()
        assert ((got - q).abs() <= 2.0 ** -4 * q.abs() * (1 + 2 * t32) + 2.0 ** -10 + 448 * 2 * t32).all()
        assert (got.abs().amax(-1)[top > 0] == 448).all()
    return h, y, s


SIZES = [(1, 1), (3, 7), (5, 8), (1, 256), (130, 256), (7, 1024), (33, 1001), (4, 2048), (3, 4096), (2, 8200), (2, 16384), (9, 130), (6, 136)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(mf, dt, quant, rows, cols):
    _norm(mf, rows, cols, dt, quant)
    _norm(mf, rows, cols, dt, quant, residual=False, eps=0.1)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("pad", [1, 4, 8])
@pytest.mark.parametrize("cols", [256, 999, 2304])
def test_row_strides(mf, dt, quant, pad, cols):
    _norm(mf, 37, cols, dt, quant, pad=pad)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("cols,pad", [(126, 0), (334, 0), (1001, 1), (1568, 2), (1570, 0), (1571, 0)])
def test_many_rows(mf, dt, quant, cols, pad):
    """Rows enough for a warp to take a whole row; rows that start on 2, 4 or 8 bytes only."""
    _norm(mf, 2500, cols, dt, quant, pad=pad)


@pytest.mark.parametrize("cols", [256, 250, 251])
def test_block_of_nan(mf, cols):
    x = torch.randn((2100, cols), device="cuda")
    x[7, 3] = -math.nan  # as a sum of squares it reaches all of the row
    w = torch.ones(cols, device="cuda")
    y, s = torch.empty((2100, cols), device="cuda", dtype=E4M3), torch.empty((2100, 2), device="cuda")
    mf.rms_norm(x, w, y, scales=s, scale_group=128)
    bad = torch.isnan(s).any(-1)
    assert bad[7] and bad.sum() == 1 and torch.isnan(y[7].float()).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("quant", ["row", "128"])
def test_zero_blocks_have_scale_one(mf, dt, quant):
    def change(x, r, w):
        x[1], r[1] = 0, 0
        x[2, 128:256], r[2, 128:256] = 0, 0
    _, y, s = _norm(mf, 4, 512, dt, quant, change=change)
    assert (s[1] == 1).all() and (y[1].float() == 0).all()
    if quant == "128":
        assert s[2, 1] == 1 and (s[2, 0] != 1)


@pytest.mark.parametrize("cols", [256, 1001, 4096])
def test_in_place(mf, cols):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x, r = (torch.randn((50, cols), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.ones(cols, device="cuda", dtype=torch.bfloat16)
    h, y = torch.empty_like(x), torch.empty_like(x)
    mf.rms_norm(x, w, y, residual=r, residual_out=h)
    a, b = x.clone(), r.clone()
    mf.rms_norm(a, w, a, residual=b, residual_out=b)
    assert torch.equal(a, y) and torch.equal(b, h)


@pytest.mark.parametrize("quant", [None, "row", "128"])
def test_nan_stays_in_its_row(mf, quant):
    x = torch.ones((3, 512), device="cuda", dtype=torch.bfloat16)
    x[1, 200] = math.nan
    w = torch.ones(512, device="cuda", dtype=torch.bfloat16)
    y = torch.empty((3, 512), device="cuda", dtype=E4M3 if quant else torch.bfloat16)
    s = torch.empty((3, {"row": 1, "128": 4}[quant]), device="cuda") if quant else None
    mf.rms_norm(x, w, y, scales=s, scale_group=128 if quant == "128" else 0)
    assert torch.isnan(y[1].float()).all() and torch.isfinite(y[0].float()).all() and torch.isfinite(y[2].float()).all()


def test_no_rows(mf):
    x = torch.empty((0, 64), device="cuda")
    mf.rms_norm(x, torch.ones(64, device="cuda"), torch.empty_like(x))


def test_refusals(mf):
    x = torch.ones((4, 256), device="cuda", dtype=torch.bfloat16)
    w, y = torch.ones(256, device="cuda", dtype=torch.bfloat16), torch.empty_like(x)
    y8, s = torch.empty((4, 256), device="cuda", dtype=E4M3), torch.empty((4, 1), device="cuda")
    big = torch.ones((5, 256), device="cuda", dtype=torch.bfloat16)
    mf.rms_norm(x, w, y8, scales=s)
    for kw, status in [
            (dict(y=y8), mf.EINVAL), (dict(scales=s), mf.EINVAL), (dict(y=y.float()), mf.EINVAL),
            (dict(y=y8, scales=s, scale_group=64), mf.EINVAL), (dict(weight=w.float()), mf.EINVAL),
            (dict(weight=w[:255]), mf.EINVAL), (dict(eps=-1.0), mf.EINVAL), (dict(eps=math.inf), mf.EINVAL),
            (dict(residual=x[:3]), mf.EINVAL), (dict(residual=x.t().contiguous().t()), mf.EINVAL),
            (dict(x=x.half()), mf.EINVAL), (dict(residual_out=y), mf.EINVAL),
            (dict(x=big[:4], y=big[1:]), mf.EINVAL), (dict(y=x.cpu()), mf.EINVAL)]:
        with pytest.raises(mf.MafatError) as e:
            mf.rms_norm(**{**dict(x=x, weight=w, y=y), **kw})
        assert e.value.status == status, kw
    wide = torch.ones((1, 16392), device="cuda")
    with pytest.raises(mf.MafatError) as e:
        mf.rms_norm(wide, wide[0], torch.empty_like(wide))
    assert e.value.status == mf.EUNSUPPORTED
    torch.cuda.synchronize()
