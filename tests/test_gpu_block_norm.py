"""The norms around a block against their definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _block(mf, rows, cols, dt, quant=None, post=True, gates=1, want="hy", pad=0, branch=0.75, keep=1.5, eps=1e-6, seed=1,
           change=None, in_place=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rows_of(fill=None, t=dt, n=rows):
        b = torch.empty((n, cols + pad), dtype=t, device="cuda")[:, :cols]
        return b if fill is None else b.copy_(fill)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    x, r = rows_of(randn(rows, cols) * 2), rows_of(randn(rows, cols))
    w1, w2 = ((1 + 0.3 * randn(cols)).to(dt) for _ in range(2))
    gate = rows_of(randn(gates, cols), n=gates) if gates else None
    if change:
        change(x, r)
    # in 64 bits, with how far fp32 may be from it: a sum of cols squares in pieces as of the norm alone, root, division and
    # products of 2^-24 each
    t32, u = (cols / 32 + 32) * 2.0 ** -24, 2.0 ** -24
    n64 = x.double()
    rel = 0.0
    if post:
        n64, rel = n64 / torch.sqrt(n64.square().mean(-1, keepdim=True) + eps) * w1.double(), t32
    if gates:
        n64, rel = n64 * gate.double().repeat_interleave(rows // gates, 0), rel + u
    h64 = keep * r.double() + branch * n64
    off = branch * n64.abs() * (rel + 2 * u) + abs(keep) * r.double().abs() * u + h64.abs() * u  # of h
    rms = torch.sqrt(h64.square().mean(-1, keepdim=True) + eps)
    y64 = h64 / rms * w2.double()
    off_y = off / rms * w2.double().abs() + y64.abs() * (off.square().mean(-1, keepdim=True).sqrt() / rms + t32)

    h = rows_of() if "h" in want else None
    y = rows_of(t=E4M3 if quant else dt) if "y" in want else None
    if in_place:
        h, y = {"h=r": (r, y), "h=x": (x, y), "y=x": (h, x), "h=r,y=x": (r, x)}[in_place]
    s = torch.empty((rows, 1 if quant == "row" else -(-cols // 128)), device="cuda") if quant else None
    mf.block_norm(x, r, h, post_weight=w1 if post else None, gate=gate if gates != 1 else gate[0].contiguous() if gates else None,
                  branch_scale=branch, residual_scale=keep, weight=w2 if y is not None else None, y=y, scales=s,
                  scale_group=128 if quant == "128" else 0, eps=eps)
    out = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24  # half a step of 8 or 24 significant bits
    if h is not None:
        assert ((h.double() - h64).abs() <= off + out * (h64.abs() + off) + 1e-37).all()
    if y is None:
        return h, y, s
    if not quant:
        assert ((y.double() - y64).abs() <= off_y + out * (y64.abs() + off_y) + 1e-37).all()
        return h, y, s
    width = cols if quant == "row" else 128
    for i in range(s.shape[1]):
        b, e = (z[:, i * width:(i + 1) * width] for z in (y64, off_y))
        top, slack = b.abs().amax(-1), e.amax(-1)
        want_s = torch.where(top == 0, torch.ones_like(top), top / 448)
        assert ((s[:, i].double() - want_s).abs() <= slack / 448 + 2.0 ** -23 * want_s).all()
        # 8 bits: half of 1/8 of the power of two below a value (2^-4 of it), or of the smallest step 2^-9
        got = y[:, i * width:(i + 1) * width].float().double() * s[:, i:i + 1].double()
        assert ((got - b).abs() <= 2.0 ** -4 * b.abs() * (1 + 2.0 ** -20) + 2.0 ** -10 * want_s[:, None] + 3 * e + 2.0 ** -20 * top[:, None]).all()
    return h, y, s


SIZES = [(1, 1), (3, 7), (6, 8), (2, 256), (130, 256), (8, 1024), (33, 1001), (4, 2048), (3, 4096), (2, 8200), (2, 16384), (9, 130), (6, 136)]
BOTH = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dt", BOTH)
@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(mf, dt, quant, rows, cols):
    _block(mf, rows, cols, dt, quant)
    _block(mf, rows, cols, dt, quant, post=False, gates=rows, eps=0.1)
    _block(mf, rows, cols, dt, quant, gates=0, keep=0.0)


@pytest.mark.parametrize("dt", BOTH)
@pytest.mark.parametrize("want", ["h", "y", "hy"])
@pytest.mark.parametrize("rows,gates", [(12, 3), (12, 12), (3000, 3), (3000, 1500), (2500, 1)])
@pytest.mark.parametrize("cols", [96, 1568])
def test_gates_and_what_is_wanted(mf, dt, want, rows, gates, cols):
    _block(mf, rows, cols, dt, want=want, gates=gates)


@pytest.mark.parametrize("dt", BOTH)
@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("cols,pad", [(126, 0), (256, 1), (334, 0), (999, 4), (1001, 1), (1568, 2), (1570, 0), (1571, 0), (2304, 8)])
@pytest.mark.parametrize("rows", [37, 2500])
def test_strides_and_many_rows(mf, dt, quant, cols, pad, rows):
    _block(mf, rows, cols, dt, quant, pad=pad)


@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("cols,pad", [(4, 0), (132, 0), (484, 4), (1000, 12), (2060, 0), (4900, 4), (16380, 0)])
@pytest.mark.parametrize("rows", [3, 2100])
def test_rows_of_whole_accesses_of_four(mf, quant, cols, pad, rows):
    _block(mf, min(rows, 8000000 // cols), cols, torch.bfloat16, quant, pad=pad, gates=1)


@pytest.mark.parametrize("dt", BOTH)
@pytest.mark.parametrize("quant", [None, "row", "128"])
@pytest.mark.parametrize("rows,cols", [(600, 2048), (1030, 600), (1030, 512), (1023, 1024), (300, 4096), (1500, 1312), (150, 16384)])
def test_rows_of_few_and_of_many_warps(mf, dt, quant, rows, cols):
    _block(mf, rows, cols, dt, quant, gates=rows)


@pytest.mark.parametrize("dt", BOTH)
@pytest.mark.parametrize("how", ["h=r", "h=x", "y=x", "h=r,y=x"])
@pytest.mark.parametrize("rows,cols", [(5, 5000), (2100, 512)])
def test_in_place(mf, dt, how, rows, cols):
    _block(mf, rows, cols, dt, in_place=how)


def test_values_at_the_ends(mf):
    """Zeros, a row whose squares vanish beside eps, one whose squares pass fp32's range (its norm is 0), NaN in one row."""
    x, r = torch.randn((6, 512), device="cuda"), torch.randn((6, 512), device="cuda")
    x[0], r[0], x[1], x[2], x[3, 7] = 0, 0, x[1] * 1e-25, x[2] * 1e25, math.nan
    w = torch.ones(512, device="cuda")
    h, y = torch.empty_like(x), torch.empty_like(x)
    mf.block_norm(x, r, h, post_weight=w, weight=w, y=y)
    assert not h[0].any() and not y[0].any() and torch.equal(h[2], r[2])
    assert torch.isnan(h[3]).all() and torch.isnan(y[3]).all() and torch.isfinite(y[[0, 1, 2, 4, 5]]).all()
    x[4] = r[4] * 0 + 1e25
    mf.block_norm(x, r, h, weight=w, y=y)
    assert not y[4].any() and torch.isfinite(h[4]).all()


def test_no_rows(mf):
    z = torch.empty((0, 64), device="cuda")
    mf.block_norm(z, z, torch.empty_like(z), post_weight=torch.ones(64, device="cuda"), weight=torch.ones(64, device="cuda"), y=torch.empty_like(z))
