"""Attention from its definition in 64 bits, with bounds on the error of an fp32 (or bf16 x
bf16 -> fp32) implementation, derived from the inputs.

A score is a sum of 128 products: its rounding errors add up like a random walk, at six
sigma 6 sqrt(128) u sum|q_d k_d| with u = 2^-24 (round to nearest) or 2^-23 (tensor cores,
which truncate). A score off by e moves a probability by the factor exp(e), so the output
moves by at most 2 e E with E = sum_j p_j |v_j|; sums over n keys add n u' E at most. Where
probabilities are rounded to bf16 (8 significant bits) for the product with V, another
2^-8 E; a bf16 output is within 2^-8 of itself."""
import math

import torch

DH = 128


def attend(q, k, v, hidden, scale, dtype, tc):
    """One head: q [n, 128], k, v [m, 128], hidden [n, m]. Returns out, lse (64 bits) and the
    bounds on their errors."""
    qd, kd, vd = q.double(), k.double(), v.double()
    n, m = hidden.shape
    if m == 0:
        z = torch.zeros(n, DH, dtype=torch.float64, device=q.device)
        return z, torch.full((n,), -math.inf, dtype=torch.float64, device=q.device), z, z[:, 0]
    x = qd @ kd.T * scale
    x[hidden] = -math.inf
    lse = torch.logsumexp(x, 1)
    none = hidden.all(1)
    p = torch.where(hidden, 0.0, torch.exp(x - torch.where(none, 0.0, lse)[:, None]))
    u = 2.0 ** -23 if tc else 2.0 ** -24
    walk = (qd.abs() @ kd.abs().T * scale).masked_fill(hidden, 0.0).amax(1) * 6 * math.sqrt(DH) * u + 2.0 ** -21
    E = p @ vd.abs()
    bound = E * (2 * walk + (m + 16) * u + (2.0 ** -8 if tc else 0.0))[:, None]
    out = p @ vd
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (out.abs() + bound)
    return out, lse, bound + 1e-30, walk + (m + 16) * u + torch.where(none, 0.0, lse.abs()) * 2.0 ** -22


def check(out, lse, ref, what):
    o, l, bo, bl = ref
    err = (out.double() - o).abs()
    assert torch.isfinite(out).all(), f"{what}: not finite"
    assert (err <= bo).all(), f"{what}: out off by {float((err / bo).max()):.3g} of its bound"
    empty = o.new_tensor(0.0) + (l == -math.inf)
    assert torch.equal(lse == -math.inf, l == -math.inf), f"{what}: empty rows differ"
    lerr = torch.where(empty > 0, 0.0, (lse.double() - torch.where(empty > 0, 0.0, l)).abs())
    assert (lerr <= bl).all(), f"{what}: lse off by {float((lerr / bl).max()):.3g} of its bound"


def hidden_mask(lq, lk, prefix, causal, device):
    """[lq, prefix + lk]: which keys row i does not see"""
    h = torch.zeros(lq, prefix + lk, dtype=torch.bool, device=device)
    if causal:
        i, j = torch.arange(lq, device=device)[:, None], torch.arange(lk, device=device)[None]
        h[:, prefix:] = j > i + lk - lq
    return h
