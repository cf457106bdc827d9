"""What the example's drafting form takes for the prompt and for the answer, and that it keeps drafts that are right."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROMPT = 9


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("answer_frames", os.path.join(ROOT, "examples", "answer_frames.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def states(example):
    return example.frame_states(1)


@pytest.fixture()
def adjusted(example, monkeypatch):
    """The logits of each call, before and after."""
    calls, real = [], example.mf.adjust_logits

    def record(logits, out, **kw):
        before = logits.clone()
        real(logits, out, **kw)
        calls.append((before, out.clone()))
    monkeypatch.setattr(example.mf, "adjust_logits", record)
    return calls


def _decoder(example, states, requests, nodes):
    d = example.DraftingDecoder(1, requests, states.shape[1], states.shape[2], room=60, nodes=nodes)
    d.read_frames(states)
    return d


def _expected(d, before, r, row, answer):
    """A row's logits by the definition, in 64 bits, and the sizes that its roundings are relative to."""
    x = before[r, row].double().cpu()
    n, said = torch.zeros_like(x), torch.zeros_like(x, dtype=torch.bool)
    for t in answer:
        n[t] += 1
    said[answer] = True
    said[d.given[r].tolist()] = True
    rep, f = d.repetition[r].double().item(), d.frequency[r].double().item()
    y = torch.where(said, torch.where(x > 0, x / rep, x * rep), x)
    return y - f * n, y.abs() + 2 * f * n


@pytest.mark.parametrize("nodes", [1, 7])
def test_the_prompt_is_no_answer(example, states, adjusted, nodes):
    """Its tokens are said, but only those that came after count as repeated; of the prompt one row a request is adjusted."""
    d = _decoder(example, states, 2, nodes)
    d.given = torch.tensor([[5, 5, 5, 7, 8, 9, 5, 7, 11], [0, 1, 2, 3, 4, 5, 6, 7, 8]], device="cuda")
    last = d.read_prompt(d.given)
    assert adjusted[0][0].shape[1] == 1 and d.prompt.tolist() == [PROMPT] * 2
    answer = [[], []]

    def check(ways):
        before, after = adjusted[-1]
        for r in range(2):
            assert len(ways[r]) == before.shape[1]
            for row, way in enumerate(ways[r]):
                want, size = _expected(d, before, r, row, answer[r] + way)
                # the quotient or product, frequency times count, the difference
                off = (after[r, row].double().cpu() - want).abs()
                assert (off <= 2.0 ** -24 * (size + want.abs()) * 1.01).all(), (r, row)
    check([[[]], [[]]])
    for _ in range(4):
        tokens, kept = [last], d.length.clone()
        for j in range(1, nodes):
            tokens.append(d.next_tokens[tokens[d.parents[j]], (j - 1) % 2])
        t, n, last = d.step(last)
        assert torch.equal(d.length, kept + n.to(torch.int32)) and d.prompt.tolist() == [PROMPT] * 2
        ways = [[], []]
        for r in range(2):
            for j in range(nodes):
                way, k = [], j
                while k >= 0:
                    way.append(int(tokens[k][r]))
                    k = d.parents[k]
                ways[r].append(way)
        check(ways)
        for r in range(2):
            answer[r] += [int(tokens[0][r])] + t[r, :int(n[r]) - 1].tolist()
            assert d.said[r, PROMPT:int(d.length[r])].tolist() == answer[r]


def test_right_drafts_are_kept(example, states, adjusted):
    """A drafter that is told what the decoder will ask for has all its drafts kept, in a tree's one step as in steps of a token each: the
    tokens, their places, histories and caches.  Requests are chosen by the steps of a token alone: no token with two
    successors, and logits whose first is ahead of the second by more than the two forms' roundings."""
    requests = 12
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    prompt = torch.randint(0, 1000, (requests, PROMPT), generator=g, device="cuda")
    one, many = _decoder(example, states, requests, 1), _decoder(example, states, requests, 7)
    last, first = one.read_prompt(prompt), many.read_prompt(prompt)
    assert torch.equal(last, first) and torch.equal(one.length, many.length)
    chain, ahead = [last], []
    for _ in range(3):
        t, n, last = one.step(last)
        assert (n == 1).all()
        chain.append(t[:, 0])
        two = adjusted[-1][1][:, 0].topk(2).values
        ahead.append((two[:, 0] - two[:, 1]) / adjusted[-1][1][:, 0].abs().amax(-1))
    chain, ahead = torch.stack(chain, 1).tolist(), torch.stack(ahead, 1).amin(-1).tolist()
    follows, chosen = {}, []
    for r in range(requests):
        pairs = dict(zip(chain[r], chain[r][1:]))
        if len(set(chain[r])) == 4 and ahead[r] > 0.02 and all(follows.get(x, y) == y for x, y in pairs.items()):
            follows.update(pairs)
            chosen.append(r)
    assert chosen, ahead
    for x, y in follows.items():
        many.next_tokens[x, 0] = y
    before = many.length.clone()
    t, n, last = many.step(first)
    assert torch.equal(many.length, before + n.to(torch.int32))
    for r in chosen:
        assert int(n[r]) == 3 and t[r].tolist() == chain[r][1:] and int(last[r]) == chain[r][3], r
        assert many.said[r, PROMPT:PROMPT + 3].tolist() == chain[r][:3] and torch.equal(many.said[r, :PROMPT + 3], one.said[r, :PROMPT + 3])
        for cm, co in zip(many.cache, one.cache):
            x, y = cm[:, r, PROMPT:PROMPT + 3].float(), co[:, r, PROMPT:PROMPT + 3].float()
            assert (x - y).abs().max() <= 0.05 * y.abs().max(), r
