"""A small decoder that answers over frames, from the image to the next tokens.

The CNN front-end turns each frame into a feature map, NHWC, which is a sequence of H * W states.  A
decoder of random weights then reads them: its self-attention layers have the frame's states as a
prefix that all requests about the frame share, its cross-attention layers look at the states
beside the text, and a norm with the residual's addition stands before each.  The last norm comes out in
8 bits with a scale a row.  The prompts of all requests go through at once, then single tokens.

With --draft each step verifies a tree of drafted tokens instead of taking one: rotary positions, attention of the tree to the
frame and the request's cache, norms on both sides of a gated block, and logits with penalties for what was said.

    python examples/answer_frames.py [--frames 2] [--requests 4] [--prompt 13] [--steps 8] [--draft 7]

Products with weight matrices are torch's; everything else is the framework's.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2107_06960_gb300 as mf  # noqa: E402
import synth  # noqa: E402

BF16 = torch.bfloat16


class Decoder:
    """`layers` pairs of self-attention (over the frame and the request's own tokens) and
    cross-attention (over the frame), `requests` requests for each of `frames` frames."""

    def __init__(self, frames, requests, n_states, channels, room, width=512, heads=8, heads_kv=2, dim=64, layers=2,
                 vocab=1000, seed=0):
        self.frames, self.requests, self.n_states, self.room = frames, requests, n_states, room
        self.width, self.heads, self.heads_kv, self.dim, self.layers = width, heads, heads_kv, dim, layers
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def w(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") / rows ** 0.5).to(BF16)

        kv = 2 * heads_kv * dim
        self.embedding = w(vocab, width) * vocab ** 0.5
        self.state_kv = [(w(channels, kv), w(channels, kv)) for _ in range(layers)]
        self.self_in = [w(width, heads * dim + kv) for _ in range(layers)]
        self.cross_in = [w(width, heads * dim) for _ in range(layers)]
        self.out = [(w(heads * dim, width), w(heads * dim, width)) for _ in range(layers)]
        self.gain = [torch.ones(width, device="cuda", dtype=BF16) for _ in range(2 * layers + 1)]
        self.state_gain = torch.ones(channels, device="cuda", dtype=BF16)
        self.head = w(width, vocab)
        self.batch = frames * requests
        self.cache = [torch.zeros(2, self.batch, room, heads_kv, dim, device="cuda", dtype=BF16) for _ in range(layers)]
        self.length = torch.zeros(self.batch, device="cuda", dtype=torch.int32)
        self.plans = {}

    def plan(self, kind, n_q):
        """One plan for each kind of attention and number of tokens in a call.  Queries, keys and values are
        read where the products left them: side by side."""
        if (kind, n_q) not in self.plans:
            shape = (self.heads, self.heads_kv, self.dim)
            side, both = (self.heads + 2 * self.heads_kv) * self.dim, 2 * self.heads_kv * self.dim
            kv = (self.n_states * both, both, self.dim)
            self.plans[kind, n_q] = (
                mf.PrefixAttention(self.frames, self.requests, n_q, self.n_states, self.room, *shape,
                                   q_strides=(n_q * side, side, self.dim), prefix_k_strides=kv, prefix_v_strides=kv)
                if kind == "self" else
                mf.CrossAttention(self.frames, self.requests * n_q, self.n_states, *shape, k_strides=kv, v_strides=kv))
        return self.plans[kind, n_q]

    def read_frames(self, states):
        """states [frames][n_states][channels]: their keys and values for every layer, once for all requests."""
        flat = states.reshape(-1, states.shape[-1])
        y = torch.empty_like(flat)
        mf.rms_norm(flat, self.state_gain, y)
        shape = (self.frames, self.n_states, 2, self.heads_kv, self.dim)
        self.states = [[(y @ m).view(shape).unbind(2) for m in pair] for pair in self.state_kv]

    def norm(self, x, residual, i):
        h, y = torch.empty_like(x), torch.empty_like(x)
        mf.rms_norm(x, self.gain[i], y, residual=residual, residual_out=h)
        return h, y

    def forward(self, tokens):
        """tokens [batch][n_q], the next ones of every request: logits of the last, [batch][vocab]."""
        n_q = tokens.shape[1]
        at = self.length[:, None].long() + torch.arange(n_q, device="cuda")
        self.length += n_q
        x, h = self.embedding[tokens.reshape(-1)], torch.zeros(tokens.numel(), self.width, device="cuda", dtype=BF16)
        q_cols = self.heads * self.dim
        for i in range(self.layers):
            h, y = self.norm(x, h, 2 * i)
            qkv = y @ self.self_in[i]
            q = qkv.view(self.batch, n_q, -1, self.dim)[:, :, :self.heads]
            kv = qkv[:, q_cols:].view(self.batch, n_q, 2, self.heads_kv, self.dim)
            rows = torch.arange(self.batch, device="cuda")[:, None]
            self.cache[i][0][rows, at], self.cache[i][1][rows, at] = kv[:, :, 0], kv[:, :, 1]
            o = torch.empty(q.shape, device="cuda", dtype=BF16)
            self.plan("self", n_q).run(q, *self.states[i][0], *self.cache[i], o, own_len=self.length)
            x = o.view(-1, q_cols) @ self.out[i][0]
            h, y = self.norm(x, h, 2 * i + 1)
            # the requests of a frame are neighbours: their tokens are one sequence of queries to its states
            q = (y @ self.cross_in[i]).view(self.frames, self.requests * n_q, self.heads, self.dim)
            o = torch.empty_like(q)
            self.plan("cross", n_q).run(q, *self.states[i][1], o)
            x = o.view(-1, q_cols) @ self.out[i][1]
        last = torch.arange(n_q - 1, tokens.numel(), n_q, device="cuda")
        x, h = x[last], h[last]
        y = torch.empty(x.shape, device="cuda", dtype=torch.float8_e4m3fn)
        scales = torch.empty(x.shape[0], 1, device="cuda")
        mf.rms_norm(x, self.gain[-1], y, residual=h, scales=scales)
        return (y.to(BF16) @ self.head).float() * scales  # an 8-bit product would take y and its scales as they are


def tree_words(parents):
    """Words of a tree's ways from the root, [1][n][ceil(n / 32)], for parents before their children."""
    n = len(parents)
    way = torch.zeros(n, n, dtype=torch.bool)
    for j, parent in enumerate(parents):
        if parent >= 0:
            way[j] = way[parent]
        way[j, j] = True
    way = torch.nn.functional.pad(way.long(), (0, -n % 32)).view(n, -1, 32)
    words = (way << torch.arange(32)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)[None].cuda()


class DraftingDecoder(Decoder):
    """Each step reads a tree of `nodes` drafted tokens of every request, whose root is the last token taken, and keeps those
    on the way that its logits agree with.  Here the drafts are what follows a token by embedding and head alone."""

    def __init__(self, *args, nodes=7, **kw):
        super().__init__(*args, **kw)
        self.nodes = nodes
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        self.after_gain = [torch.ones(self.width, device="cuda", dtype=BF16) for _ in range(2 * self.layers)]
        self.gate = [(1 + 0.1 * torch.randn(self.width, generator=g, device="cuda")).to(BF16) for _ in range(2 * self.layers)]
        self.rotary = mf.Rotary(self.dim, scaling=mf.ROTARY_BLEND, factor=2.0, first_positions=1024)
        self.next_tokens = (self.embedding.float() @ self.head.float()).topk(2).indices
        self.parents = [(j + 1) // 2 - 1 for j in range(nodes)]  # two children a node
        self.ways = tree_words(self.parents)
        self.said = torch.zeros(self.batch, self.room, device="cuda", dtype=torch.int32)
        self.prompt = torch.zeros(self.batch, device="cuda", dtype=torch.int32)  # how much of it is the prompt
        self.repetition = torch.full((self.batch,), 1.2, device="cuda")
        self.frequency = torch.full((self.batch,), 0.1, device="cuda")

    def tree_plan(self, n_q):
        if ("tree", n_q) not in self.plans:
            side, both = (self.heads + 2 * self.heads_kv) * self.dim, 2 * self.heads_kv * self.dim
            kv = (self.n_states * both, both, self.dim)
            self.plans["tree", n_q] = mf.TreeAttention(self.frames, self.requests, n_q, self.n_states, self.room, self.heads, self.heads_kv,
                                                       self.dim, q_strides=(n_q * side, side, self.dim), prefix_k_strides=kv,
                                                       prefix_v_strides=kv)
        return self.plans["tree", n_q]

    def between(self, x, residual, i):
        """The norm behind block i - 1 and its gate, the residual's addition, the norm before block i."""
        h, y = torch.empty_like(x), torch.empty_like(x)
        behind = {} if i == 0 else dict(post_weight=self.after_gain[i - 1], gate=self.gate[i - 1], residual_scale=0.95)
        mf.block_norm(x, residual, h, weight=self.gain[i], y=y, **behind)
        return h, y

    def read_tree(self, tokens, ways, positions):
        """tokens, positions [batch][n], a tree behind self.length tokens of each request: what stands before the head, [batch][n][width]."""
        n = tokens.shape[1]
        places = self.length[:, None] + torch.arange(n, device="cuda", dtype=torch.int32)
        x = self.embedding[tokens.reshape(-1)]
        h, q_cols = torch.zeros_like(x), self.heads * self.dim
        for i in range(self.layers):
            h, y = self.between(x, h, 2 * i)
            qkv = (y @ self.self_in[i]).view(self.batch, n, -1, self.dim)
            q, k, v = qkv.split([self.heads, self.heads_kv, self.heads_kv], 2)
            self.rotary.run(positions, q=q, q_out=q, k=k, k_out=self.cache[i][0], v=v, v_out=self.cache[i][1], places=places)
            o = torch.empty(q.shape, device="cuda", dtype=BF16)
            self.tree_plan(n).run(q, *self.states[i][0], *self.cache[i], ways, o, own_len=self.length + n)
            x = o.view(-1, q_cols) @ self.out[i][0]
            h, y = self.between(x, h, 2 * i + 1)
            q = (y @ self.cross_in[i]).view(self.frames, self.requests * n, self.heads, self.dim)
            o = torch.empty_like(q)
            self.plan("cross", n).run(q, *self.states[i][1], o)
            x = o.view(-1, q_cols) @ self.out[i][1]
        return self.between(x, h, 2 * self.layers)[1].view(self.batch, n, -1)

    def adjusted(self, y, **drafted):
        """Logits of y [batch][n][width], with penalties for what was said, fp32.  drafted: what each row has besides."""
        logits = y @ self.head
        out = torch.empty(logits.shape, device="cuda")
        mf.adjust_logits(logits, out, tokens=self.said, lengths=self.length, prompt_lengths=self.prompt, repetition=self.repetition,
                         frequency=self.frequency, **drafted)
        return out

    def keep(self, tokens, path, count):
        """The first count [batch] nodes of each path [batch][n] become the request's next tokens."""
        n, rows = path.shape[1], torch.arange(self.batch, device="cuda")[:, None]
        at = self.length[:, None].long() + torch.arange(n, device="cuda")
        for c in self.cache:
            c[:, rows, at] = c[:, rows, self.length[:, None].long() + path]
        self.said[rows, at] = tokens.gather(1, path).to(torch.int32)
        self.length += count.to(torch.int32)

    def read_prompt(self, tokens):
        n = tokens.shape[1]
        positions = torch.arange(n, device="cuda", dtype=torch.int32).expand(self.batch, n).contiguous()
        y = self.read_tree(tokens, tree_words(range(-1, n - 1)), positions)
        path = torch.arange(n, device="cuda").expand(self.batch, n)
        self.keep(tokens, path, torch.full((self.batch,), n, device="cuda"))
        self.prompt += n
        return self.adjusted(y[:, -1:])[:, 0].argmax(-1)

    def step(self, last):
        """last [batch], the token to go on from: the tokens that follow it [batch][depth], how many of them count, the new last."""
        tokens, depth = [last], [0]
        for j in range(1, self.nodes):
            tokens.append(self.next_tokens[tokens[self.parents[j]], (j - 1) % 2])
            depth.append(depth[self.parents[j]] + 1)
        tokens = torch.stack(tokens, 1)
        positions = self.length[:, None] + torch.tensor(depth, device="cuda", dtype=torch.int32)
        y = self.read_tree(tokens, self.ways, positions.contiguous())
        best = self.adjusted(y, drafts=tokens.to(torch.int32), tree=self.ways).argmax(-1)
        # down from the root, as long as a drafted child is what its parent's logits ask for
        at = torch.zeros(self.batch, device="cuda", dtype=torch.long)
        path, on = [at], torch.ones(self.batch, device="cuda", dtype=torch.bool)
        count = torch.ones(self.batch, device="cuda", dtype=torch.long)
        for _ in range(max(depth)):
            want, here = best.gather(1, at[:, None])[:, 0], at
            for child in (2 * here + 1, 2 * here + 2):
                inside = child.clamp(max=self.nodes - 1)
                hit = on & (child < self.nodes) & (tokens.gather(1, inside[:, None])[:, 0] == want) & (at == here)
                at = torch.where(hit, child, at)
            on = on & (at != here)
            count += on
            path.append(at)
        path = torch.stack(path, 1)
        taken = best.gather(1, path)  # what each node on the way asks for; the last of them is not drafted
        self.keep(tokens, path, count)
        return taken, count, taken.gather(1, count[:, None] - 1)[:, 0]


def frame_states(frames, size=224, seed=7):
    """Feature maps of random frames by the 16-layer front-end: [frames][(size / 16)^2][256]."""
    layers = synth.YOLO16
    net = mf.Net(layers, size, size, 3)
    net.set_params(synth.make_params(layers, 3, seed, "bf16"))
    plan = mf.Plan(net, cut=8, grids=[(2, 2), (1, 1)], batch=frames)
    image = torch.from_numpy(synth.make_input(frames, size, size, 3, seed, "bf16")).to(BF16).cuda()
    _, _, _, h, w, c = net.shape(len(layers) - 1)
    states = torch.empty(frames, h, w, c, device="cuda", dtype=BF16)
    plan.run(image, states)
    plan.sync_status(like=image)
    return states.view(frames, h * w, c)


def answer_with_drafts(a):
    """As many tokens of each request as there are steps, or more; returns the first ones of each."""
    states = frame_states(a.frames)
    room = a.prompt + (a.steps + 1) * (a.draft.bit_length() + 1) + a.draft
    d = DraftingDecoder(a.frames, a.requests, states.shape[1], states.shape[2], room=room, nodes=a.draft)
    d.read_frames(states)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    last = d.read_prompt(torch.randint(0, d.embedding.shape[0], (d.batch, a.prompt), generator=g, device="cuda"))
    answers, kept = [[int(x)] for x in last], 0
    for _ in range(a.steps - 1):
        tokens, count, last = d.step(last)
        kept += int(count.sum())
        for answer, row, n in zip(answers, tokens.tolist(), count.tolist()):
            answer.extend(row[:n])
    for plan in d.plans.values():
        plan.sync_status(like=last)
    print("%.2f tokens of a request a step" % (kept / max(1, (a.steps - 1) * d.batch)))
    for n, row in enumerate(answers):
        print("frame %d, request %d: %s" % (n // a.requests, n % a.requests, " ".join(map(str, row))))
    return torch.tensor([row[:a.steps] for row in answers])


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--frames", type=int, default=2)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=13)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--draft", type=int, default=0, help="nodes of a tree of drafted tokens, 0: none")
    a = ap.parse_args(argv)
    if a.draft:
        return answer_with_drafts(a)
    states = frame_states(a.frames)
    d = Decoder(a.frames, a.requests, states.shape[1], states.shape[2], room=a.prompt + a.steps)
    d.read_frames(states)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tokens = torch.randint(0, d.embedding.shape[0], (d.batch, a.prompt), generator=g, device="cuda")
    got = []
    for step in range(a.steps):
        if step == 1:  # the prompts are read, plans and libraries set up
            torch.cuda.synchronize()
            began = time.perf_counter()
        tokens = d.forward(tokens).argmax(-1, keepdim=True)
        got.append(tokens)
    answer = torch.cat(got, 1).cpu()
    if a.steps > 1:
        print("%.2f ms a step of %d requests" % ((time.perf_counter() - began) * 1e3 / (a.steps - 1), d.batch))
    for plan in d.plans.values():
        plan.sync_status(like=tokens)
    for n, row in enumerate(answer.tolist()):
        print("frame %d, request %d: %s" % (n // a.requests, n % a.requests, " ".join(map(str, row))))
    return answer


if __name__ == "__main__":
    main()
