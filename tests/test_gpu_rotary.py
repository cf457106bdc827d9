"""Rotary positions against their definition: angles by exact fractions, products in 64 bits."""
import math
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
# A sine or cosine: the fraction of a turn in fp32 (2^-25 of half a turn) and in 2^-32, the function (2 ulp of values up to 1),
# and the magnitude's product and rounding.
TRIG = math.pi * 2.0 ** -25 + 2 * math.pi * 2.0 ** -32 + 2 * 2.0 ** -24 + 2 * 2.0 ** -24


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _turned(x, positions, f, m, rot, interleaved):
    """x [B][T][H][D] turned in 64 bits, and |a| + |b| of each channel's pair, times m."""
    angle = torch.tensor([[[float(p * Fraction(w) % TWO_PI) for w in f] for p in row] for row in positions.tolist()],
                         dtype=torch.float64).cuda()
    cos, sin = (m * torch.cos(angle))[:, :, None], (m * torch.sin(angle))[:, :, None]
    x = x.double()
    y, mag = x.clone(), torch.zeros_like(x)
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    mag[..., first] = mag[..., second] = m * (a.abs() + b.abs())
    return y, mag


def _check(got, x, positions, f, m, rot, interleaved, what):
    ref, mag = _turned(x, positions, f, m, rot, interleaved)
    out = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    fp32 = mag * (TRIG + 2 * 2.0 ** -24)  # and two products and a sum
    off = (got.double() - ref).abs()
    assert (off <= fp32 + out * (ref.abs() + fp32)).all(), what
    assert torch.equal(got[..., rot:], x[..., rot:]), what


def _rotary(mf, B, T, H, Hk, D, dtype, rot=0, interleaved=False, room=None, far=5000, side=True, seed=1, what="qkv", **kw):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = torch.bfloat16 if dtype == mf.BF16 else torch.float32
    both = torch.randn((B, T, H + 2 * Hk, D), generator=g, device="cuda").to(dt)
    q, k, v = both[:, :, :H], both[:, :, H:H + Hk], both[:, :, H + Hk:]
    if not side:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    positions = torch.randint(0, far, (B, T), generator=g, device="cuda").to(torch.int32)
    plan = mf.Rotary(D, rot, dtype=dtype, interleaved=interleaved, **kw)
    f, m = plan.frequencies()
    rot = rot or D
    q_out = torch.full((B, T, H, D), math.nan, dtype=dt, device="cuda")
    n = room or T
    k_out = torch.randn((B, n, Hk, D), generator=g, device="cuda").to(dt)
    v_out = torch.randn((B, n, Hk, D), generator=g, device="cuda").to(dt)
    was_k, was_v = k_out.clone(), v_out.clone()
    places = None
    if room:  # any order, some of the tokens nowhere
        places = torch.stack([torch.randperm(max(room, T), generator=g, device="cuda")[:T] for _ in range(B)]).to(torch.int32)
        places[places >= room] = 2 ** 31 - 1
        places.view(-1)[::5] = -1
    args = {}
    if "q" in what:
        args.update(q=q, q_out=q_out)
    if "k" in what:
        args.update(k=k, k_out=k_out)
    if "v" in what:
        args.update(v=v, v_out=v_out)
    plan.run(positions, places=places, **args)
    if "q" in what:
        _check(q_out, q, positions, f, m, rot, interleaved, "q")
    at = torch.arange(T, device="cuda").expand(B, T) if places is None else places.long()
    kept = torch.ones(B, n, dtype=torch.bool, device="cuda")
    for b in range(B):
        here = (at[b] >= 0) & (at[b] < n)
        kept[b, at[b][here]] = False
        if "k" in what and here.any():
            _check(k_out[b, at[b][here]][None], k[b, here][None], positions[b, here][None], f, m, rot, interleaved, "k")
        if "v" in what:
            assert torch.equal(v_out[b, at[b][here]], v[b, here])
    for name, now, was in (("k", k_out, was_k), ("v", v_out, was_v)):  # places that no token has stay
        assert torch.equal(now[kept], was[kept]) and (name in what or torch.equal(now, was))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(8, 0), (64, 0), (128, 0), (80, 40), (128, 64), (40, 38), (64, 2), (96, 12), (256, 0), (72, 70), (256, 2)])
def test_layouts(mf, dtype, interleaved, D, rot):
    _rotary(mf, 2, 5, 4, 2, D, dtype, rot, interleaved)
    _rotary(mf, 3, 2, 3, 1, D, dtype, rot, interleaved, room=9, side=False)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,T,H,Hk,room", [(1, 1, 1, 1, 1), (64, 1, 32, 8, 40), (1, 33, 9, 3, None), (5, 77, 17, 5, 100), (2, 700, 8, 2, 650), (300, 1, 5, 5, 3)])
def test_sizes(mf, dtype, B, T, H, Hk, room):
    _rotary(mf, B, T, H, Hk, 64, dtype, room=room)
    _rotary(mf, B, T, H, Hk, 128, dtype, 32, True, room=room, side=False)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("H,Hk,D,rot", [(1, 1, 64, 0), (2, 1, 64, 24), (1, 2, 40, 12), (1, 1, 8, 2), (1, 1, 256, 250)])
def test_many_tokens_of_few_heads(mf, dtype, H, Hk, D, rot):
    """As many as a block of threads takes, and a last block with few."""
    for interleaved in (False, True):
        _rotary(mf, 3, 1777, H, Hk, D, dtype, rot, interleaved, room=1800)


@pytest.mark.parametrize("what", ["q", "k", "v", "qk", "qv", "kv"])
def test_some_of_the_tensors(mf, what):
    _rotary(mf, 3, 7, 4, 2, 64, mf.BF16, what=what)
    _rotary(mf, 3, 7, 4, 2, 64, mf.BF16, room=20, what=what)


@pytest.mark.parametrize("dtype", [0, 1])
def test_scalings(mf, dtype):
    """Each by its formula."""
    for rot in (64, 20):
        plain = [10000.0 ** (-2 * i / rot) for i in range(rot // 2)]
        base = [(5e5 * 4 ** (rot / (rot - 2))) ** (-2 * i / rot) for i in range(rot // 2)]
        keep = [min(1, max(0, (4096 * f / (2 * math.pi) - 2) / (20 - 2))) for f in plain]
        for kw, f, m in ((dict(), plain, 1), (dict(scaling=mf.ROTARY_LINEAR, factor=4.0), [x / 4 for x in plain], 1),
                         (dict(scaling=mf.ROTARY_BASE, factor=4.0, base=5e5), base, 1),
                         (dict(scaling=mf.ROTARY_BLEND, factor=16.0, first_positions=4096, fast=20.0, slow=2.0),
                          [x * (w + (1 - w) / 16) for x, w in zip(plain, keep)], 0.1 * math.log(16) + 1),
                         (dict(frequencies=[(-1) ** i * 0.3 * i for i in range(rot // 2)], magnitude=2.5),
                          [(-1) ** i * 0.3 * i for i in range(rot // 2)], 2.5)):
            got, mag = mf.Rotary(64, rot, dry_run=True, **kw).frequencies()
            assert mag == pytest.approx(m, rel=1e-14) and got == pytest.approx(f, rel=1e-13)
            _rotary(mf, 2, 6, 3, 1, 64, dtype, rot, far=200000, **kw)


def test_far_and_negative_positions(mf):
    plan = mf.Rotary(64, dtype=mf.FP32)
    f, m = plan.frequencies()
    positions = torch.tensor([[0, -1, 2 ** 31 - 1, -2 ** 31, 123456789, 2 ** 24 + 1, -77777777]], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 7, 3, 64), device="cuda")
    o = torch.empty_like(q)
    plan.run(positions, q=q, q_out=o)
    _check(o, q, positions, f, m, 64, False, "far")
    assert torch.equal(o[:, 0], q[:, 0])  # position 0 turns nothing


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [64, 24])
def test_in_place(mf, interleaved, rot):
    """Queries and keys where they are, side by side in one matrix."""
    plan = mf.Rotary(64, rot, interleaved=interleaved)
    f, m = plan.frequencies()
    qkv = torch.randn((3, 11, 8, 64), device="cuda").to(torch.bfloat16)
    was = qkv.clone()
    positions = torch.arange(33, device="cuda", dtype=torch.int32).view(3, 11)
    q, k, v = qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:]
    plan.run(positions, q=q, q_out=q, k=k, k_out=k, v=v, v_out=v)
    _check(q, was[:, :, :4], positions, f, m, rot, interleaved, "q")
    _check(k, was[:, :, 4:6], positions, f, m, rot, interleaved, "k")
    assert torch.equal(v, was[:, :, 6:])


def test_turning_back(mf):
    """The gradient of a rotation is the rotation by the negative angles: with negative frequencies, against the formula's
    derivative (its transpose) and against differences."""
    f = [0.9 ** i for i in range(16)]
    there, back = mf.Rotary(40, 32, dtype=mf.FP32, frequencies=f), mf.Rotary(40, 32, dtype=mf.FP32, frequencies=[-x for x in f])
    positions = torch.tensor([[3, 1000, 99999]], dtype=torch.int32, device="cuda")
    x, dy = torch.randn((1, 3, 2, 40), device="cuda"), torch.randn((1, 3, 2, 40), device="cuda")
    y, dx, y2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    there.run(positions, q=x, q_out=y)
    back.run(positions, q=dy, q_out=dx)
    # <dy, R x> = <R^T dy, x>: sums of 240 products of rounded results
    scale = (x.abs().max() * dy.abs().max()).double() * x.numel()
    assert abs((dy.double() * y.double()).sum() - (dx.double() * x.double()).sum()) <= 4 * (TRIG + 2.0 ** -22) * scale
    step = torch.zeros_like(x)
    step[0, 1, 0, 5] = 1.0  # linear: a difference of any size is the derivative
    there.run(positions, q=x + step, q_out=y2)
    got = (dy.double() * (y2.double() - y.double())).sum()
    assert abs(got - dx[0, 1, 0, 5].double()) <= 8 * (TRIG + 2.0 ** -22) * scale


def test_nothing_to_do(mf):
    plan = mf.Rotary(64)
    z = torch.empty((0, 4, 2, 64), device="cuda", dtype=torch.bfloat16)
    plan.run(torch.empty((0, 4), device="cuda", dtype=torch.int32), q=z, q_out=torch.empty_like(z))
    k = torch.randn((2, 3, 1, 64), device="cuda").to(torch.bfloat16)
    none = torch.empty((2, 0, 1, 64), device="cuda", dtype=torch.bfloat16)
    plan.run(torch.zeros((2, 3), device="cuda", dtype=torch.int32), k=k, k_out=none, places=torch.zeros((2, 3), device="cuda", dtype=torch.int32))
