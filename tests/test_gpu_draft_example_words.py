"""What the example's drafting form takes for the prompt and for the answer."""
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
