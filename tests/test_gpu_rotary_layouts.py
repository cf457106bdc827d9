"""Rotary positions into caches that hold keys and values between one another, and in place in one matrix."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIZES = dict(b=3, w=3, t=7, h=2)


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


@pytest.mark.parametrize("order", list(itertools.permutations("bwth")))
@pytest.mark.parametrize("dt,D,rot,inter", [(torch.bfloat16, 64, 0, False), (torch.float32, 40, 10, True)])
def test_any_order(mf, order, dt, D, rot, inter):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    plan = mf.Rotary(D, rot, dtype=mf.BF16 if dt == torch.bfloat16 else mf.FP32, interleaved=inter)
    x = torch.randn([SIZES[d] for d in order] + [D], generator=g, device="cuda").to(dt)
    q, k, v = x.permute([order.index(d) for d in "wbth"] + [4]).unbind(0)
    positions = torch.randint(0, 900, (3, 7), generator=g, device="cuda").to(torch.int32)
    want = [torch.empty(t.shape, device="cuda", dtype=dt) for t in (q, k)]
    apart = [t.contiguous() for t in (q, k, v)]
    plan.run(positions, q=apart[0], q_out=want[0], k=apart[1], k_out=want[1])
    # into a cache of keys, values and what else there is
    room = 11
    cache = torch.randn([{**SIZES, "t": room}[d] for d in order] + [D], generator=g, device="cuda").to(dt)
    was = cache.clone()
    places = torch.stack([torch.randperm(room, generator=g, device="cuda")[:7] for _ in range(3)]).to(torch.int32)
    places[1, 2] = room
    ck, cv, other = cache.permute([order.index(d) for d in "wbth"] + [4]).unbind(0)
    plan.run(positions, k=apart[1], k_out=ck, v=apart[2], v_out=cv, places=places)
    wk, wv, wother = was.permute([order.index(d) for d in "wbth"] + [4]).unbind(0)
    for b in range(3):
        for t in range(7):
            if int(places[b, t]) < room:
                wk[b, places[b, t].long()], wv[b, places[b, t].long()] = want[1][b, t], apart[2][b, t]
    assert torch.equal(ck, wk) and torch.equal(cv, wv) and torch.equal(other, wother)
    # where they are
    plan.run(positions, q=q, q_out=q, k=k, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, apart[2])
