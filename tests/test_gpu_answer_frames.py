"""The example runs from images to tokens, and every call that it makes of an operator is right."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from lm_util import attention64, attention_tol, check  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def example():
    spec = importlib.util.spec_from_file_location("answer_frames", os.path.join(ROOT, "examples", "answer_frames.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_tokens_repeat(example):
    a, b = example.main(["--steps", "4"]), example.main(["--steps", "4"])
    assert a.shape == (8, 4) and torch.equal(a, b)


def test_each_call_against_its_definition(example, monkeypatch):
    """Prompts and single tokens; the calls follow one another without a wait in between."""
    mf = example.mf
    calls = []
    norm, cross, prefix = mf.rms_norm, mf.CrossAttention.run, mf.PrefixAttention.run

    def keep(kind, ins, outs):  # copies, in stream order: later calls may write over them
        calls.append((kind, [t.clone() if torch.is_tensor(t) else t for t in ins], [t.clone() for t in outs if t is not None]))

    def rms_norm(x, w, y, residual=None, residual_out=None, scales=None, **kw):
        norm(x, w, y, residual=residual, residual_out=residual_out, scales=scales, **kw)
        keep("norm", (x, w, residual), (y, residual_out, scales))

    def cross_run(self, q, k, v, out):
        cross(self, q, k, v, out)
        keep("cross", (q, k, v), (out,))

    def prefix_run(self, q, pk, pv, ok, ov, out, own_len=None):
        prefix(self, q, pk, pv, ok, ov, out, own_len=own_len)
        keep("prefix", (q, pk, pv, ok, ov, own_len), (out,))

    monkeypatch.setattr(mf, "rms_norm", rms_norm)
    monkeypatch.setattr(mf.CrossAttention, "run", cross_run)
    monkeypatch.setattr(mf.PrefixAttention, "run", prefix_run)
    example.main(["--steps", "3", "--prompt", "11", "--requests", "3"])
    assert [c[0] for c in calls].count("cross") == 6 and [c[0] for c in calls].count("prefix") == 6
    for kind, ins, outs in calls:
        if kind == "norm":
            x, w, r = ins
            h = x.double() + (0 if r is None else r.double())
            y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * w.double()
            t32 = (x.shape[1] / 32 + 32) * 2.0 ** -24  # the sum of squares and what follows, as in the norm's own tests
            if outs[0].dtype == torch.float8_e4m3fn:
                got = outs[0].float().double() * outs[-1].double()
                assert ((got - y).abs() <= 2.0 ** -4 * y.abs() + (2.0 ** -10 + 1e-3) * outs[-1].double()).all()
            else:
                assert ((outs[0].double() - y).abs() <= (2.0 ** -8 + t32) * y.abs() + 1e-37).all()
            continue
        q, k, v = ins[:3]
        for n in range(q.shape[0]):
            f = n * k.shape[0] // q.shape[0]
            segs = [(k[f], v[f], torch.ones(q.shape[1], k.shape[1], dtype=torch.bool, device="cuda"))]
            if kind == "prefix":
                ok, ov, own_len = ins[3:]
                last = own_len[n] - q.shape[1] + torch.arange(q.shape[1], device="cuda")
                segs.append((ok[n], ov[n], torch.arange(ok.shape[1], device="cuda")[None] <= last[:, None]))
            ref, _, a, mag = attention64(q[n], segs, 1 / math.sqrt(q.shape[-1]))
            keys = sum(s[0].shape[0] for s in segs)
            check(outs[0][n], ref, attention_tol(ref, a, mag, keys, q.shape[-1], True), kind)
