"""Norm, rotation, the 4-bit cache and attention over it by their definitions, in 64 bits on the CPU."""
import math

import numpy as np
import torch


def table(positions, rot, base=10000.0):
    inv = base ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(positions)[:, None] * inv
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).float()


def norm_rope(x, weight, rows, interleaved=False, eps=1e-6):
    """x [..., L, D]; rows [..., L, rot] of the table, or None.  Returns (z, |y cos| + |y' sin|)."""
    x = x.double()
    y = x if weight is None else x * weight.double() / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    if rows is None:
        return y, y.abs()
    rot = rows.shape[-1]
    cos, sin = rows[..., :rot // 2].double(), rows[..., rot // 2:].double()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    out = []
    for u, v in ((a * cos - b * sin, b * cos + a * sin), ((a * cos).abs() + (b * sin).abs(), (b * cos).abs() + (a * sin).abs())):
        z = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
        out.append(torch.cat([z, y[..., rot:] if not out else y[..., rot:].abs()], -1))
    return out[0], out[1]


def to_bf16(z):
    """One rounding from 64 bits, halves to even."""
    m, e = np.frexp(z.numpy())
    return torch.from_numpy(np.ldexp(np.rint(m * 256), e - 8)).to(torch.bfloat16)


def quantise(x):
    """bf16 x [..., D] -> (codes [..., D], steps, least values [..., D / 64]) in 64 bits"""
    y = x.double().unflatten(-1, (-1, 64))
    low, high = y.amin(-1), y.amax(-1)
    step = to_bf16((high - low) / 15).double()
    n = torch.where(step[..., None] > 0, (y - low[..., None]) / torch.where(step > 0, step, 1.0)[..., None], 0.0)
    return torch.round(n).clamp(0, 15).flatten(-2).long(), step, low


def held(x):
    n, step, low = quantise(x)
    return (n.double().unflatten(-1, (-1, 64)) * step[..., None] + low[..., None]).flatten(-2)


def unpack(blocks):
    """uint8 [..., 18 D] on the CPU -> for keys and for values: (codes [..., 16, D], steps, least values [..., 16, D / 64])"""
    D = blocks.shape[-1] // 18
    w = blocks.contiguous().numpy().view(np.uint32)
    out = []
    for values in (False, True):
        t, c = np.meshgrid(np.arange(16), np.arange(D // 8), indexing="ij")
        if values:
            h, q, e, g, j = t // 8, t // 2 % 4, t % 2, c % 8, c // 8
            lane = 4 * g + q
            at = 2 * D + ((h * 32 + lane) * 2 + e if D == 64 else ((j // 2 * 2 + h) * 32 + lane) * 4 + 2 * e + j % 2)
        else:
            at = t * (D // 8) + c % 4 * (D // 32) + c // 4
        codes = np.stack([w[..., at] >> (4 * i) & 15 for i in range(8)], -1).reshape(*w.shape[:-1], 16, D)
        pairs = w[..., 4 * D + values * D // 4:][..., :D // 4].reshape(*w.shape[:-1], 16, D // 64)
        half = [torch.from_numpy((x << 16).astype(np.uint32).view(np.float32).astype(np.float64)) for x in (pairs & 0xffff, pairs >> 16)]
        out.append((torch.from_numpy(codes.astype(np.int64)), half[0], half[1]))
    return out


def keep(q, kd):
    """q [rows, D]: indices of the kd columns of largest energy, equal ones to the lower index, ascending"""
    return torch.sort(q.double().square().sum(0).float(), descending=True, stable=True).indices[:kd].sort().values


def attention(q, K, V, n, step, low, rows, causal, kd):
    """One query head's rows q [L, D] over held keys K and values V = low + step n [T, D] (codes n, steps and least values by
    64 columns), the last `rows` tokens being the queries'.  Returns (O, how far a kernel may be from it).

    How far, per element.  Rounding of O to bf16: 2^-8 |O|.  Weights times steps in fp16: 2^-11 of each term P s n, and where they
    leave fp16's normal range 2^-25 against a largest one of 2^6 or more, times a code of up to 15, for each token.  Logits in fp32: eight
    groups of 16 products added up on the tensor cores (two roundings toward zero of 2^-23 each) and six fp32 operations, of terms
    no larger than |q| (|m| + 15 s): 2^-18 of their sum B; that, 2^-20 for the exponentials and sums, move every weight, and with
    it the normaliser."""
    L, D = q.shape
    T = K.shape[0]
    O, tol = torch.zeros(L, D, dtype=torch.float64), torch.zeros(L, D, dtype=torch.float64)
    if rows == 0 or T == 0:
        return O, tol
    idx = keep(q[:rows], kd) if kd < D else torch.arange(D)
    x = q.double()[:rows, idx] @ K[:, idx].T / math.sqrt(D)
    size = (low_k_size(K, idx) @ q.double().abs()[:rows, idx].T).T / math.sqrt(D)
    if causal:
        seen = torch.arange(T) <= torch.arange(rows)[:, None] + T - rows
        x = x.masked_fill(~seen, -math.inf)
    P = torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
    O[:rows] = P @ V
    s = step.repeat_interleave(64, -1)
    moved = 2 * (2.0 ** -18 * size.amax(-1, keepdim=True) * 1.4427 + 2.0 ** -20)
    tol[:rows] = (2.0 ** -8 * O[:rows].abs() + 2.0 ** -11 * (P @ (s * n)) + moved * (P @ (low.repeat_interleave(64, -1).abs() + s * n))
                  + T * 15 * 2.0 ** -31 * (P @ s).amax(-1, keepdim=True) + 1e-30)
    return O, tol


def low_k_size(K, idx):
    """No smaller than |m| + 15 s: twice the largest magnitude of the 64 columns, and their range."""
    y = K.unflatten(-1, (-1, 64))
    size = 3.1 * y.abs().amax(-1, keepdim=True).expand_as(y).flatten(-2)
    return size[:, idx]
