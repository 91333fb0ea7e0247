"""The 4-bit form of rows and attention over it, from their contract in include/provip.h, in plain
numpy and torch, with bounds on the error of an fp32 implementation."""
import math

import numpy as np
import torch

DH, ROW4 = 128, 72


def bf16_bits(x):
    """float32 -> bits of the nearest bf16 (ties to even), finite inputs"""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def bf16_value(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32)


def pack(rows):
    """float32 [n, 128] -> codes [n, 128] (0..15), scale bits [n, 4] uint16, operation by operation"""
    v = np.ascontiguousarray(rows, dtype=np.float32).reshape(-1, 4, 32)
    with np.errstate(all="ignore"):
        hi, lo = v.max(-1), v.min(-1)
        e = np.where(hi >= -lo, hi, lo)
        fine = np.isfinite(v).all(-1) & (np.abs(e) < 2.0 ** 100)
        bits = np.where(fine, bf16_bits(np.where(fine, e, 0) * np.float32(-0.125)), 0x7FFF).astype(np.uint16)
        bits = np.where(fine & (np.abs(e) < 2.0 ** -123), 0, bits).astype(np.uint16)
        d = bf16_value(bits)
        r = np.where(d == 0, np.float32(0), np.float32(1) / np.where(d == 0, np.float32(1), d)).astype(np.float32)
        y = np.clip(v * r[..., None], np.float32(-8), np.float32(7))
        n = np.where(fine[..., None], np.rint(np.where(fine[..., None], y, 0)) + 8, 0).astype(np.int64)
    return n.reshape(-1, DH), bits


def place(value):
    """(byte, shift) of value 32 q + 4 g + t in a row's codes"""
    q, g, t = value // 32, value % 32 // 4, value % 4
    return 2 * (4 * g + q) + t // 2, 4 * (t % 2)


BYTE = torch.tensor([place(i)[0] for i in range(DH)])
SHIFT = torch.tensor([place(i)[1] for i in range(DH)])


def row_bytes(pages, page_size, slot, h):
    """codes [64] and scale bits [4] of one head's row (a CPU uint8 pool)"""
    page, row = slot // page_size, slot % page_size
    block = pages[page, h].numpy()
    return block[row * 64:row * 64 + 64], block[page_size * 64 + row * 8:page_size * 64 + row * 8 + 8].view(np.uint16)


def put(pages, page_size, slot, h, codes, bits):
    """one head's row into a CPU uint8 pool"""
    page, row = slot // page_size, slot % page_size
    out = np.zeros(64, dtype=np.uint8)
    for i in range(DH):
        at, shift = place(i)
        out[at] |= int(codes[i]) << shift
    pages[page, h, row * 64:row * 64 + 64] = torch.from_numpy(out)
    pages[page, h, page_size * 64 + row * 8:page_size * 64 + row * 8 + 8] = torch.from_numpy(bits.view(np.uint8).copy())


def values(pages, page_size, slots):
    """what the rows at slots stand for, [n, H, 128] in 64 bits (any device)"""
    dev, H = pages.device, pages.shape[1]
    slots = slots.long()
    page, row = slots // page_size, slots % page_size
    block = pages[page]  # [n, H, page_size * 72]
    at = (row[:, None] * 64 + BYTE.to(dev))[:, None].expand(-1, H, -1)
    n = (block.gather(2, at).long() >> SHIFT.to(dev)) & 15
    low = (page_size * 64 + row[:, None] * 8 + 2 * (torch.arange(DH, device=dev) // 32))[:, None].expand(-1, H, -1)
    bits = (block.gather(2, low).int() << 16) | (block.gather(2, low + 1).int() << 24)
    return (n - 8).double() * bits.view(torch.float32).double()


def random_pool(g, n_pages, page_size, H, device, spread=1.0):
    """A pool of random codes and scales of either sign around 0.3 * spread (a factor of four apart)."""
    codes = torch.randint(0, 256, (n_pages, H, page_size * 64), generator=g, device=device, dtype=torch.uint8)
    d = spread * torch.exp2(torch.rand(n_pages, H, page_size * 4, generator=g, device=device) * 2 - 2.7)
    d = d * (1 - 2 * torch.randint(0, 2, d.shape, generator=g, device=device))
    return torch.cat([codes, d.to(torch.bfloat16).view(torch.uint8).view(n_pages, H, page_size * 8)], 2)


def attend(q, k, v, scale, dtype):
    """One row of a head: q [128], k, v [m, 128] in 64 bits (values unrounded). Returns out, lse and bounds on
    their errors.

    A score is four group sums of 32 products (exact in fp32: a bf16 query, or a third of an fp32 one, times
    a code), each times its scale: sums of n terms in the tensor cores truncate, 2^-23 each, so at six sigma
    of a walk 6 sqrt(128) 2^-23 sum|q k|; fp32 queries split into three bf16 leave 2^-24 of each product. A
    score off by e moves a weight by exp(e), the output by 2 e E with E = sum p |v| (and the same of the
    magnitudes of codes times weights). A weight times a scale is rounded to bf16 (2^-8 of it), for fp32 to 24
    bits and products' sums of a step again to 2^-23; sums over m keys add m 2^-23 E at most; weights by
    ex2.approx are off by 2^-22; a bf16 output is within 2^-8 of itself."""
    if k.shape[0] == 0:
        z = torch.zeros(DH, dtype=torch.float64, device=q.device)
        return z, torch.tensor(-math.inf, dtype=torch.float64, device=q.device), z, z[0]
    qd = q.double()
    x = k @ qd * scale
    lse = torch.logsumexp(x, 0)
    p = torch.exp(x - lse)
    u, m = 2.0 ** -23, k.shape[0]
    walk = float((k.abs() @ qd.abs() * scale).max()) * 6 * math.sqrt(DH) * u + float(x.abs().max()) * 2.0 ** -22 + 2.0 ** -21
    E, out = p @ v.abs(), p @ v
    low = dtype == torch.bfloat16
    bound = E * (2 * walk + (m + 16) * u + (2.0 ** -8 if low else 0.0))
    if low:
        bound = bound + 2.0 ** -8 * (out.abs() + bound)
    return out, lse, bound + 1e-30, walk + (m + 16) * u + abs(float(lse)) * 2.0 ** -22


def turn(x, pos, freq, axis, w, eps, factor):
    """norm and rotation of x [T, H, 128] in 64 bits, pos [axes, T]: the result, and what an fp32
    implementation may be off by before its last rounding.

    Sine and cosine: 2 ulp (2^-22), of an angle off by its rounding to fp32, pi 2^-24, and 2^-33 turns:
    2^-21 in all. Norm: a sum of 128 squares in a chain of 19, half its 19 2^-24 in the root, a root of 2 ulp
    and three products: 2^-20. Products and their sum: 2^-23. Together 2^-19 of |a| + |b|."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    at = torch.stack([pos[a].double() * f for a, f in zip(axis, freq)], 1)[:, None]
    a, b = y[..., :64], y[..., 64:]
    c, s = torch.cos(at), torch.sin(at)
    size = (a.abs() + b.abs()) * abs(factor) * 2.0 ** -19
    return torch.cat([a * c - b * s, b * c + a * s], -1) * factor, torch.cat([size, size], -1)
