"""A step of a decoder that verifies drafted tokens: the operators one after another, as they are used, against their
definitions; captured and replayed on new data; and on other streams."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from draft_util import random_ways, seen_own, words  # noqa: E402
from lm_util import attention64, attention_tol, check  # noqa: E402

FRAMES, REQUESTS, NODES, STATES, ROOM, HEADS, KV, DIM, WIDTH, VOCAB = 2, 3, 9, 196, 60, 8, 2, 64, 512, 1000


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


class Step:
    """One layer and the logits, in bf16; a request's committed tokens and its tree change from step to step."""

    def __init__(self, mf, seed=0):
        self.mf = mf
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def w(*shape):
            return (torch.randn(shape, generator=g, device="cuda") / shape[0] ** 0.5).to(torch.bfloat16)
        n = FRAMES * REQUESTS
        self.n, self.embedding = n, w(VOCAB, WIDTH) * VOCAB ** 0.5
        self.qkv, self.out, self.head = w(WIDTH, (HEADS + 2 * KV) * DIM), w(HEADS * DIM, WIDTH), w(WIDTH, VOCAB)
        self.gains = [(1 + 0.1 * torch.randn(WIDTH, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(3)]
        self.gate = w(1, WIDTH)[0]
        self.states = [torch.randn((FRAMES, STATES, KV, DIM), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
        self.cache = [torch.randn((n, ROOM, KV, DIM), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
        side = (HEADS + 2 * KV) * DIM
        self.rotary = mf.Rotary(DIM, scaling=mf.ROTARY_BLEND, factor=4.0, first_positions=2048)
        self.tree = mf.TreeAttention(FRAMES, REQUESTS, NODES, STATES, ROOM, HEADS, KV, DIM, q_strides=(NODES * side, side, DIM))
        self.repetition, self.presence, self.frequency = (torch.full((n,), x, device="cuda") for x in (1.3, 0.2, 0.1))
        self.io = None

    def data(self, seed):
        """The step's inputs, in buffers that stay."""
        g = torch.Generator()
        g.manual_seed(seed)
        n = self.n
        nodes = torch.randint(1, NODES + 1, (n,), generator=g)
        before = torch.randint(0, ROOM - NODES + 1, (n,), generator=g)
        way = random_ways(n, NODES, seed)
        depth = way.sum(-1) - 1
        places = before[:, None] + torch.arange(NODES)
        places[torch.arange(NODES)[None] >= nodes[:, None]] = -1
        said = torch.randint(0, VOCAB, (n, ROOM), generator=g)
        masks = torch.rand((4, VOCAB), generator=g) < 0.7
        new = {"drafts": torch.randint(0, VOCAB, (n, NODES), generator=g), "nodes": nodes, "own_len": before + nodes, "way": words(way),
               "positions": 5000 + before[:, None] + depth, "places": places, "said": said, "lengths": before,
               "masks": words(masks), "mask_rows": torch.randint(-1, 4, (n, NODES), generator=g)}
        new = {k: v.to(torch.int32).cuda() for k, v in new.items()}
        if self.io is None:
            self.io = new
        for k, v in new.items():
            self.io[k].copy_(v)
        self.host = {"nodes": nodes.tolist(), "own_len": (before + nodes).tolist(), "way": way}

    def run(self):
        mf, io, n = self.mf, self.io, self.n
        x = self.embedding[io["drafts"].view(-1).long()]
        h, y = torch.empty_like(x), torch.empty_like(x)
        zero = torch.zeros_like(x)
        mf.block_norm(x, zero, h, weight=self.gains[0], y=y)
        qkv = (y @ self.qkv).view(n, NODES, HEADS + 2 * KV, DIM)
        was = qkv.clone()
        q, k, v = qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV], qkv[:, :, HEADS + KV:]
        self.rotary.run(io["positions"], q=q, q_out=q, k=k, k_out=self.cache[0], v=v, v_out=self.cache[1], places=io["places"])
        o = torch.empty((n, NODES, HEADS, DIM), device="cuda", dtype=torch.bfloat16)
        self.tree.run(q, *self.states, *self.cache, io["way"], o, nodes=io["nodes"], own_len=io["own_len"])
        x = o.view(-1, HEADS * DIM) @ self.out
        h2, y2 = torch.empty_like(h), torch.empty_like(h)
        mf.block_norm(x, h, h2, post_weight=self.gains[1], gate=self.gate, branch_scale=0.8, residual_scale=1.1, weight=self.gains[2], y=y2)
        logits = (y2 @ self.head).view(n, NODES, VOCAB)
        adjusted = torch.empty((n, NODES, VOCAB), device="cuda")
        mf.adjust_logits(logits, adjusted, tokens=io["said"], lengths=io["lengths"], repetition=self.repetition, presence=self.presence,
                         frequency=self.frequency, drafts=io["drafts"], tree=io["way"], masks=io["masks"], mask_rows=io["mask_rows"])
        return {"x0": self.embedding[io["drafts"].view(-1).long()], "h": h, "y": y, "was": was, "q": q, "k": self.cache[0], "v": self.cache[1],
                "o": o, "x": x, "h2": h2, "y2": y2, "logits": logits, "adjusted": adjusted}

    def check(self, r):
        """Each operator's results from what it was given."""
        half = 2.0 ** -8
        t32 = (WIDTH / 32 + 32) * 2.0 ** -24

        def norm(h, w):
            return h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * w.double()
        assert torch.equal(r["h"], r["x0"])
        y = norm(r["x0"].double(), self.gains[0])
        assert ((r["y"].double() - y).abs() <= (half + t32) * y.abs() + 1e-37).all()
        branch = 0.8 * norm(r["x"].double(), self.gains[1]) * self.gate.double()
        h = 1.1 * r["h"].double() + branch
        off = (branch.abs() + 1.1 * r["h"].double().abs()) * (t32 + 4 * 2.0 ** -24)
        assert ((r["h2"].double() - h).abs() <= half * h.abs() + 2 * off).all()
        y = norm(h, self.gains[2])
        assert ((r["y2"].double() - y).abs() <= half * y.abs() + 4 * (off / h.square().mean(-1, keepdim=True).sqrt() + t32 * y.abs())).all()
        # positions: angles in 64 bits are good to 2^-53 of some thousands of radians
        f, m = self.rotary.frequencies()
        angle = self.io["positions"].double()[..., None] * torch.tensor(f, dtype=torch.float64, device="cuda")
        cos, sin = (m * torch.cos(angle))[:, :, None], (m * torch.sin(angle))[:, :, None]

        def turned(x):
            a, b = x.double().split(DIM // 2, -1)
            return torch.cat([a * cos - b * sin, a * sin + b * cos], -1), m * torch.cat([a.abs() + b.abs()] * 2, -1) * 2.0 ** -20
        ref, fp32 = turned(r["was"][:, :, :HEADS])
        assert ((r["q"].double() - ref).abs() <= half * ref.abs() + 2 * fp32).all()
        ref, fp32 = turned(r["was"][:, :, HEADS:HEADS + KV])
        for b in range(self.n):
            n, end = self.host["nodes"][b], self.host["own_len"][b]
            assert ((r["k"][b, end - n:end].double() - ref[b, :n]).abs() <= half * ref[b, :n].abs() + 2 * fp32[b, :n]).all()
            assert torch.equal(r["v"][b, end - n:end], r["was"][b, :n, HEADS + KV:])
            seen = seen_own(self.host["way"][b], end, n, NODES, ROOM).cuda()
            live = (torch.arange(NODES, device="cuda") < n)[:, None].expand(-1, STATES)
            segs = [(self.states[0][b // REQUESTS], self.states[1][b // REQUESTS], live), (r["k"][b], r["v"][b], seen)]
            out, _, a, mag = attention64(r["q"][b], segs, 1 / math.sqrt(DIM))
            check(r["o"][b], out, attention_tol(out, a, mag, STATES + ROOM, DIM, True), "o")
        # every row's history: what the request has said, and the way to the node
        for b in range(self.n):
            for t in range(NODES):
                ids = self.io["said"][b, :int(self.io["lengths"][b])].tolist() + self.io["drafts"][b].cpu()[self.host["way"][b, t]].tolist()
                count = torch.bincount(torch.tensor(ids), minlength=VOCAB).double().cuda()
                x = r["logits"][b, t].double()
                rep = float(self.repetition[b])
                y = torch.where(count > 0, torch.where(x > 0, x / rep, x * rep), x)
                y = y - float(self.frequency[b]) * count - float(self.presence[b]) * (count > 0)
                row = int(self.io["mask_rows"][b, t])
                if row >= 0:
                    bits = torch.tensor([(w >> i) & 1 for w in self.io["masks"][row].tolist() for i in range(32)][:VOCAB], device="cuda")
                    y = torch.where(bits > 0, y, torch.full_like(y, -math.inf))
                got = r["adjusted"][b, t].double()
                assert torch.equal(got == -math.inf, y == -math.inf)
                fine = y != -math.inf
                size = x.abs() * rep + 2 * count
                assert ((got - y).abs()[fine] <= (6 * 2.0 ** -24 * size)[fine] + 1e-37).all()


def test_steps(mf):
    s = Step(mf)
    for seed in range(3):
        s.data(seed)
        s.check(s.run())
    s.tree.sync_status(like=s.cache[0])


def test_captured_and_replayed(mf):
    """A graph of the step, replayed on other trees, lengths and histories, gives what the calls give; a second graph of
    the same plans is replayed between."""
    s = Step(mf)
    s.data(0)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s.run()  # libraries set up
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                r = s.run()
            graphs.append((g, r))
        for seed in (5, 6, 7):
            s.data(seed)
            cache = [c.clone() for c in s.cache]
            for g, r in graphs:
                for c, was in zip(s.cache, cache):
                    c.copy_(was)
                g.replay()
                torch.cuda.synchronize()
                s.check(r)
                got = {k: v.clone() for k, v in r.items()}
                for c, was in zip(s.cache, cache):
                    c.copy_(was)
                want = s.run()
                torch.cuda.synchronize()
                for k in ("h", "y", "q", "k", "v", "o"):  # what no library product rounds in its own order
                    assert torch.equal(got[k], want[k]), k


def test_two_streams_at_once(mf):
    """Two programs with plans of their own."""
    steps = [Step(mf, seed) for seed in (1, 2)]
    streams = [torch.cuda.Stream() for _ in steps]
    for s in steps:
        s.data(9)
    torch.cuda.synchronize()
    results = []
    for _ in range(4):
        results = []
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                results.append(s.run())
    torch.cuda.synchronize()
    for s, r in zip(steps, results):
        s.check(r)
