"""The example's drafting form runs, repeats, and takes a token or more of every request in each step."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("answer_frames", os.path.join(ROOT, "examples", "answer_frames.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("nodes", [1, 2, 7, 40])
def test_runs_and_repeats(example, nodes):
    args = ["--steps", "5", "--draft", str(nodes), "--requests", "3", "--prompt", "11"]
    a, b = example.main(args), example.main(args)
    assert a.shape == (6, 5) and torch.equal(a, b) and (a >= 0).all() and (a < 1000).all()


def test_what_is_kept(example):
    """Drafts that are right by construction are all kept: their places, histories and caches are those of tokens taken one by
    one, and so is what follows (the two decoders' logits differ by roundings alone)."""
    states = example.frame_states(1)
    make = lambda nodes: example.DraftingDecoder(1, 2, states.shape[1], states.shape[2], room=60, nodes=nodes)  # noqa: E731
    one, many = make(1), make(7)
    prompt = torch.arange(18, device="cuda").view(2, 9) % 1000
    for d in (one, many):
        d.read_frames(states)
    a, b = one.read_prompt(prompt), many.read_prompt(prompt)
    assert torch.equal(a, b) and torch.equal(one.length, many.length)
    taken, last = [], a
    for _ in range(4):
        t, n, last = one.step(last)
        assert (n == 1).all()
        taken.append(t[:, 0])
    # the drafter is told what comes: each token's successor stands first, others second
    for r in range(2):
        chain = [int(a[r])] + [int(t[r]) for t in taken]
        for x, y in zip(chain, chain[1:]):
            many.next_tokens[x, 0] = y
    before = many.length.clone()
    t, n, last_many = many.step(b)
    for r in range(2):
        chain = [int(x[r]) for x in taken]
        got = t[r, :int(n[r])].tolist()
        if len(set([int(a[r])] + chain[:3])) == 4 and got[:3] == chain[:3]:
            assert int(n[r]) == 3 and int(last_many[r]) == got[2]
            assert torch.equal(many.said[r, 9:12], one.said[r, 9:12])
            for cm, co in zip(many.cache, one.cache):
                x, y = cm[:, r, 9:12].float(), co[:, r, 9:12].float()
                assert (x - y).abs().max() <= 0.05 * y.abs().max()
    assert torch.equal(many.length, before + n.to(torch.int32))
