"""Plain 64-bit implementations of the operators of a cache held in 4 bits,
written from their definitions in include/spike_proj.h: on the CPU, no code of
the library."""
import math

import numpy as np
import torch

CODES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
# scale byte -> scale: 5 exponent bits (bias 15), 3 mantissa bits; 226 is 10240
SCALES = torch.tensor([i / 8 * 2.0 ** -14 if i < 8 else (1 + i % 8 / 8) * 2.0 ** (i // 8 - 15) for i in range(227)],
                      dtype=torch.float64)


def nearest(x, table):
    """Index of the nearest number of a rising table, the even one of two as near."""
    i = torch.searchsorted(table, x).clamp(1, len(table) - 1)
    below, above = x - table[i - 1], table[i] - x
    return torch.where((below < above) | ((below == above) & (i % 2 == 1)), i - 1, i)


def quantise(x):
    """Rows [..., D] of a 16-bit type: codes, scales (uint8) and values (float64)."""
    groups = x.double().unflatten(-1, (x.shape[-1] // 16, 16))
    fine = torch.isfinite(groups).all(-1)
    a = torch.where(fine, groups.abs().amax(-1), 0.0)
    byte = nearest(a / 6, SCALES)
    s = SCALES[byte].unsqueeze(-1)
    some = fine.unsqueeze(-1) & (s > 0)
    code = nearest(torch.where(some, groups.abs() / s, 0.0), CODES)
    minus = torch.signbit(groups)
    value = torch.where(some, CODES[code] * s * torch.where(minus, -1.0, 1.0), 0.0)
    value = torch.where(fine.unsqueeze(-1), value, math.nan).flatten(-2)
    code = torch.where(some, code + 8 * minus, 0).flatten(-2)
    byte = torch.where(fine, byte, 255)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), byte.to(torch.uint8), value


def values(codes, scales):
    """What rows of codes and scales stand for, in float64."""
    code = torch.stack([codes.long() % 16, codes.long() // 16], -1).flatten(-2)
    v = CODES[code % 8] * torch.where(code < 8, 1.0, -1.0).double()
    s = torch.cat([SCALES, torch.full((29,), math.nan, dtype=torch.float64)])
    s[227:248] = torch.tensor([(1 + i % 8 / 8) * 2.0 ** (i // 8 - 15) for i in range(227, 248)], dtype=torch.float64)
    s[248] = math.inf
    return (v.unflatten(-1, (scales.shape[-1], 16)) * s[scales.long()].unsqueeze(-1)).flatten(-2)


def attend(q, k, v, lens, causal=True, scale=None, other=None):
    """CPU tensors q [B, T, Hq, D], k and v [B, C, Hkv, D] in float64, other = (out,
    lse) or None.  Returns out, lse and bounds of their errors.

    A score is an FP32 sum of D exact products: its error is at most size * (D + 8) *
    2^-23 with size = scale * sum_d |q_d k_d| (any order, truncating adders), and
    what bringing q to half precision loses.  Exponentials, the scaling of scores
    and merges are off by a few 2^-22 and 2^-23 of the exponent; sums over n entries
    by (n / 16 + 64) 2^-23.  Probabilities are rounded to half precision (2^-11, below
    the normal ones 2^-35 of the largest), and the sum that they are divided by too;
    the result is rounded once more."""
    B, T, Hq, D = q.shape
    C, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else float(np.float32(scale))
    u = torch.finfo(q.dtype).eps / 2
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64)
    tol = torch.zeros(B, T, Hq, D, dtype=torch.float64)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros(B, T, Hq, dtype=torch.float64)
    for b in range(B):
        n = min(max(int(lens[b]), 0), C)
        for h in range(Hkv):
            for t in range(T):
                far = max(0, n - (T - 1 - t)) if causal else n
                rows = slice(h * G, (h + 1) * G)
                x, keys, vals = q[b, t, rows].double(), k[b, :far, h], v[b, :far, h]
                o, l = torch.zeros(G, D, dtype=torch.float64), torch.full((G,), -math.inf, dtype=torch.float64)
                mass, ds, top = o.clone(), torch.zeros(G, dtype=torch.float64), 0.0
                if far:
                    s = scale * (x @ keys.T)
                    a = torch.softmax(s, 1)
                    o, l, mass = a @ vals, torch.logsumexp(s, 1), a @ vals.abs()
                    size = scale * (x.abs() @ keys.abs().T).amax(1)
                    lost = scale * x.abs().amax(1) * keys.abs().sum(1).max() * 2.0 ** -38
                    ds = size * (D + 8) * 2.0 ** -23 + lost + 2.0 ** -19
                    top = vals.abs().max()
                adds = (far / 16 + 64) * 2.0 ** -23
                e = mass * (2 * 2.0 ** -11 + 2 * ds.unsqueeze(1) + 2 * adds) + far * 2.0 ** -35 * top
                le = ds + adds
                if other is not None:
                    oo, ol = other[0][b, t, rows].double(), other[1][b, t, rows].double()
                    both = torch.logaddexp(l, ol)
                    wl, wo = torch.exp(l - both).nan_to_num(0), torch.exp(ol - both).nan_to_num(0)
                    big = torch.where(l == -math.inf, 0.0, l.abs()) + torch.where(ol == -math.inf, 0.0, ol.abs())
                    de = (2.0 ** -20 + big * 2.0 ** -22 + le).unsqueeze(1)       # of a weight, relative
                    oo = torch.where((wo > 0).unsqueeze(1), oo, 0.0)
                    e = wl.unsqueeze(1) * e + de * (wl.unsqueeze(1) * o.abs() + wo.unsqueeze(1) * oo.abs())
                    o = wl.unsqueeze(1) * o + wo.unsqueeze(1) * oo
                    l, le = both, le + de.squeeze(1)
                out[b, t, rows], lse[b, t, rows] = o, l
                # (half precision's own subnormals)
                tol[b, t, rows] = e + u * (o.abs() + e) + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)
                lse_tol[b, t, rows] = le + 2.0 ** -22 * torch.where(l == -math.inf, 0.0, l.abs())
    return out, lse, tol, lse_tol
