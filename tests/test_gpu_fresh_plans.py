"""Plans that are run at once, on a stream that nothing else has used."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def test_rotary(mf):
    """A plan's first run has all its frequencies: it is what the same plan does later, and turned by each plan's own angles."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((2, 64, 4, 256), generator=g, device="cuda")
    positions = torch.randint(0, 1000, (2, 64), generator=g, device="cuda").to(torch.int32)
    torch.cuda.synchronize()
    for i in range(20):
        f = [(i + 1) * 0.01 * 0.97 ** j for j in range(128)]
        first, later = torch.empty_like(x), torch.empty_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            plan = mf.Rotary(256, dtype=mf.FP32, frequencies=f)
            plan.run(positions, q=x, q_out=first)
        torch.cuda.synchronize()
        plan.run(positions, q=x, q_out=later)
        assert torch.equal(first, later)
        angle = positions[..., None, None].double() * torch.tensor(f, dtype=torch.float64, device="cuda")
        a, b = x.double().split(128, -1)
        want = torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)
        # sine and cosine: the fraction of a turn in fp32 (pi 2^-25) and in 2^-32 (2 pi 2^-32), the function (2 ulp); two products and a
        # sum (2 2^-24) of |a| + |b|; the result's rounding.  The angle in 64 bits: 1000 * 0.2 * 2^-52, nothing.
        bound = (3.15 * 2.0 ** -25 + 6.3 * 2.0 ** -32 + 4 * 2.0 ** -24 + 2 * 2.0 ** -24) * (a.abs() + b.abs())
        assert ((first.double() - want).abs() <= torch.cat([bound, bound], -1) + 2.0 ** -24 * want.abs()).all()
