"""The language operators' definitions in 64 bits, and how far a kernel's result may be from them."""
import math

import torch


def attention64(q, segs, scale):
    """q [T][H][D] of one request; segs: (k [S][Hk][D], v, seen bool [T][S]) for each set of keys.
    Returns out [T][H][D], lse [T][H], and sum_s w_s |v_s| and the largest sum_d |q_d k_d| * scale,
    which the error bounds need."""
    T, H, D = q.shape
    k = torch.cat([s[0] for s in segs]).double()
    v = torch.cat([s[1] for s in segs]).double()
    seen = torch.cat([s[2] for s in segs], 1)
    any_key = seen.any(0)
    k = torch.where(any_key[:, None, None], k, torch.zeros_like(k))  # what no query reads may be anything
    v = torch.where(any_key[:, None, None], v, torch.zeros_like(v))
    rep = H // k.shape[1] if k.shape[1] else 1
    k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    z = torch.einsum("thd,shd->ths", q.double(), k) * scale
    mag = torch.einsum("thd,shd->ths", q.double().abs(), k.abs()) * scale
    z = torch.where(seen[:, None], z, torch.full_like(z, -math.inf))
    lse = torch.logsumexp(z, -1) if z.shape[-1] else torch.full((T, H), -math.inf, dtype=torch.float64, device=q.device)
    w = torch.where(seen[:, None], torch.exp(z - torch.where(lse.isinf(), torch.zeros_like(lse), lse)[..., None]),
                    torch.zeros_like(z))
    out = torch.einsum("ths,shd->thd", w, v)
    a = torch.einsum("ths,shd->thd", w, v.abs())
    m = torch.where(seen[:, None], mag, torch.zeros_like(mag)).amax().item() if mag.numel() else 0.0
    return out, lse, a, m


def attention_tol(ref, a, mag, n, dim, bf16):
    """How far out may be from ref, from the arithmetic that the header promises.

    A score is a sum of dim products in fp32: off by (dim + 4) 2^-24 of the sum of their magnitudes
    (its scaling and the maximum's subtraction included), which moves a weight by that share, once
    in the numerator and once in the denominator.  Sums over n keys and over parts in fp32, the
    exponential (2^-22) and the division add (n + 64) 2^-23.  With bf16 the weights are rounded to
    bf16, 8 significant bits, before their product with v (2^-8 of a, the weighted magnitudes), and
    so is the result (2^-8 of it)."""
    share = 2 * (dim + 4) * 2.0 ** -24 * mag + (n + 64) * 2.0 ** -23
    tol = share * a
    if bf16:
        tol = tol + 2.0 ** -8 * (1 + 2 * share) * a + 2.0 ** -8 * (1 + share) * (ref.abs() + 2.0 ** -8 * a)
    return tol + 1e-37


def lse_tol(lse, mag, n, dim):
    """The scores' error, and that of a sum over n and of the logarithm."""
    return (dim + 4) * 2.0 ** -24 * mag + (n + 64) * 2.0 ** -23 + 2.0 ** -22 * lse.abs()


def check(got, ref, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), "%s: not finite" % what
    off = (got - ref).abs()
    worst = (off / tol).max().item() if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g of the tolerance" % (what, worst)


def check_lse(got, ref, tol, what):
    got = got.double()
    assert torch.equal(got == -math.inf, ref == -math.inf), "%s: empty rows" % what
    fine = ref != -math.inf
    check(got[fine], ref[fine], tol[fine] if torch.is_tensor(tol) else tol, what)
