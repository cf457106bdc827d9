"""Trees of drafted tokens for the tests: random ones, their words, and what a node reads."""
import torch


def random_ways(n, n_q, seed=0, free=0.15):
    """[n][n_q][n_q]: whether node j is on the way from the root to node t, t itself among them (host)."""
    g = torch.Generator()
    g.manual_seed(seed)
    way = torch.zeros(n, n_q, n_q, dtype=torch.bool)
    for b in range(n):
        for t in range(n_q):
            if t > 0 and torch.rand((), generator=g) >= free:
                way[b, t] = way[b, int(torch.randint(0, t, (), generator=g))]
            way[b, t, t] = True
    return way


def words(flags):
    """[...][n] truth values as [...][ceil(n / 32)] int32, the first in the lowest bit (host)."""
    n = flags.shape[-1]
    pad = torch.zeros(flags.shape[:-1] + (-n % 32,), dtype=torch.bool)
    x = torch.cat([flags, pad], -1).reshape(flags.shape[:-1] + (-1, 32)).long()
    x = (x << torch.arange(32)).sum(-1)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def seen_own(way, own_len, nodes, n_q, n_own):
    """[n_q][n_own]: what each node of one request reads of its own keys, from the definition."""
    own_len, nodes = min(max(own_len, 0), n_own), min(max(nodes, 0), n_q)
    seen = torch.zeros(n_q, n_own, dtype=torch.bool)
    for t in range(nodes):
        for s in range(own_len):
            j = s - (own_len - nodes)
            seen[t, s] = j < 0 or bool(way[t, j])
    return seen
