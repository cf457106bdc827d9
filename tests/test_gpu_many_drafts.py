"""adjust_logits with more drafts of a request than a tree tends to have: a prompt read as one chain, wide trees."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from draft_util import random_ways, words  # noqa: E402
from test_gpu_adjust_logits import _logits, mf  # noqa: E402,F401

F32, B16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32), (B16, B16), (B16, F32)]


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("drafts", ["chain", "tree"])
@pytest.mark.parametrize("T,V", [(128, 500), (129, 500), (129, 37), (161, 9000), (300, 700)])
def test_counts(mf, dt, out_dt, drafts, T, V):  # noqa: F811
    _logits(mf, 1 if T > 200 else 2, T, V, dt, out_dt, room=40, lengths=[40, 7][:1 if T > 200 else 2], drafts=drafts)


@pytest.mark.parametrize("dt,out_dt", TYPES)
@pytest.mark.parametrize("drafts", ["chain", "tree"])
@pytest.mark.parametrize("shared", [False, True])
def test_with_all_else(mf, dt, out_dt, drafts, shared):  # noqa: F811
    _logits(mf, 1, 130, 1100, dt, out_dt, room=2100, n_bias=9, n_masks=4, drafts=drafts, shared=(shared, shared), pad=(8, 3))
    _logits(mf, 2, 140, 333, dt, out_dt, n_bias=3, n_masks=2, drafts=drafts, shared=(shared, False), pad=(3, 0), room=5, prompts=[2, 4])
    _logits(mf, 1, 131, 5000, dt, dt, room=20, n_masks=3, drafts=drafts, in_place=True)
    _logits(mf, 2, 150, 500, dt, dt, drafts=drafts, in_place=True)


@pytest.mark.parametrize("n,bits", [(2048, "tree"), (2048, "any"), (2049, "any"), (2900, "any")])
def test_wide_trees(mf, n, bits):  # noqa: F811
    """All of a request's counts at once: the ways times the drafts' tokens, whole numbers."""
    V, f = 300, torch.tensor([0.5], device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    drafts = torch.randint(-5, V + 5, (1, n), generator=g, device="cuda").to(torch.int32)
    way = random_ways(1, n, n) if bits == "tree" else torch.rand((1, n, n), generator=g, device="cuda").cpu() < 0.5
    x = torch.randn((1, n, V), generator=g, device="cuda")
    out = torch.empty_like(x)
    mf.adjust_logits(x, out, drafts=drafts, tree=words(way).cuda(), frequency=f)
    of = torch.nn.functional.one_hot(drafts[0].long().clamp(-1, V) + 1, V + 2)[:, 1:-1].double()
    counts = way[0].cuda().double() @ of
    want = x[0].double() - 0.5 * counts  # products are exact, the difference is rounded
    assert counts.max() > (1 if bits == "tree" else 8) and ((out[0].double() - want).abs() <= 2.0 ** -24 * want.abs()).all()


def _us(call):
    for _ in range(2):
        call()
    times = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return min(times)


def test_a_prompt_as_a_chain(mf):  # noqa: F811
    """Drafts cost about what as long a history does, whose tokens every row has to write too: a row's counts are not made anew for each of
    its tokens, by going over all drafts."""
    n, V = 4096, 8192
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((1, n, V), generator=g, device="cuda").to(B16)
    out = torch.empty_like(x)
    ids = torch.randperm(V, generator=g, device="cuda")[None, :n].to(torch.int32)
    rep = torch.full((1,), 1.3, device="cuda")
    history = _us(lambda: mf.adjust_logits(x, out, tokens=ids, repetition=rep))
    chain = _us(lambda: mf.adjust_logits(x, out, drafts=ids, repetition=rep))
    said = torch.zeros((n, V), dtype=torch.bool, device="cuda")
    said[:, ids[0].long()] = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    r = x[0].float()
    want = torch.where(said, torch.where(r > 0, r / rep, r * rep), r)
    assert torch.equal(out[0], want.to(B16))
    assert chain <= 6 * history, (chain, history)
