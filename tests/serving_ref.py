"""Plain 64-bit implementations of the cache and verification operators, written
from their definitions in include/spike_proj.h: loops over sequences, heads and
query tokens on the CPU, no code of the library."""
import math

import numpy as np
import torch

# Half the unit roundoff of the types: what a rounding is off by on average.  (The
# largest is twice that; what the probabilities' errors have in common cancels
# in the division by the sum of the rounded ones.)
ROUND = {torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}


def attend(q, k, v, lens, prefix_k=None, prefix_v=None, scale=None):
    """CPU tensors as spike_proj_cache_attend takes them.  Returns out, lse,
    weights in float64 and, for error bounds, sum_j p_j |v_j| per output and
    scale * max_j sum_d |q_d k_jd| per row."""
    B, T, Hq, D = q.shape
    C, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else float(np.float32(scale))
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64)
    mass = torch.zeros(B, T, Hq, D, dtype=torch.float64)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64)
    size = torch.zeros(B, T, Hq, dtype=torch.float64)
    weights = torch.zeros(B, Hkv, C, dtype=torch.float64)
    P = 0 if prefix_k is None else prefix_k.shape[0]
    for b in range(B):
        n = min(max(int(lens[b]), 0), C)
        for h in range(Hkv):
            keys, vals = k[b, :n, h].double(), v[b, :n, h].double()
            if P:
                keys = torch.cat([prefix_k[:, h].double(), keys])
                vals = torch.cat([prefix_v[:, h].double(), vals])
            for t in range(T):
                far = P + max(0, n - (T - 1 - t))
                if far == 0:
                    continue
                rows = q[b, t, h * G:(h + 1) * G].double()
                s = scale * (rows @ keys[:far].T)
                a = torch.softmax(s, 1)
                sl = slice(h * G, (h + 1) * G)
                out[b, t, sl] = a @ vals[:far]
                mass[b, t, sl] = a @ vals[:far].abs()
                lse[b, t, sl] = torch.logsumexp(s, 1)
                size[b, t, sl] = scale * (rows.abs() @ keys[:far].abs().T).amax(1)
                weights[b, h, :far - P] += a[:, P:].sum(0)
    return out, lse, weights, mass, size


def attend_bounds(dtype, D, keys, mass, size, out, vmax):
    """Error bounds from the arithmetic that the header states.  A score is an
    FP32 sum of D exact products: its error is at most size * (D + 8) * 2^-23
    (any order, truncating adders); exponentials, running sums and their
    merges add a few 2^-22.  A probability's relative error is twice the
    score's, plus the rounding to the type (and 2^-35 of the largest one, where
    a half-precision value is subnormal); the result is rounded once more."""
    u = ROUND[dtype]
    ds = size * (D + 8) * 2.0 ** -23 + 2.0 ** -19
    lse_tol = ds + 2.0 ** -20
    out_tol = u * out.abs() * (1 + u) + mass * (u + 2 * ds.unsqueeze(-1)) + keys * 2.0 ** -35 * vmax
    if dtype == torch.float16:
        out_tol = out_tol + 2.0 ** -25          # the result's own subnormals
    return out_tol, lse_tol, 2 * ds


def evict(weights, pos, n, now, budget, recent):
    """One (sequence, head): source slot of each slot of the result."""
    if n <= budget:
        return list(range(n))

    def order(j):
        w = float(weights[j])
        if int(pos[j]) >= int(now) - recent:
            return (0, 0.0, j)
        return (1, -math.inf, j) if math.isnan(w) else (2, -w, j)
    kept = set(sorted(range(n), key=order)[:budget])
    late = sorted(j for j in kept if j >= budget)
    return [j if j in kept else late.pop(0) for j in range(budget)]


def verify(p, q, draft, u, u_sample, n_draft):
    """numpy float32 arrays of one sequence: (n, tokens), in whole numbers."""
    T, V = p.shape[0] - 1, p.shape[1]
    one = np.float32(1 - 2.0 ** -24)

    def unit(x):
        return np.float32(0) if not x > 0 else min(np.float32(x), one)

    def whole(r):
        r = np.where(r > 0, np.minimum(r, np.float32(1)), 0).astype(np.float64)     # NaN > 0 is false
        return [int(x) for x in np.rint(r * 2.0 ** 36)]

    n = 0
    while n < n_draft:
        x = int(draft[n])
        if not 0 <= x < V or not np.float32(unit(u[n]) * q[n, x]) < p[n, x]:
            break
        n += 1
    tokens = [int(x) for x in draft[:n]]
    w = whole(p[n] - q[n] if n < n_draft else p[n])
    if sum(w) == 0:
        w = whole(p[n])
    token = -1
    if sum(w):
        bound = int(float(unit(u_sample)) * 2 ** 24) * sum(w) // 2 ** 24
        run = 0
        for token, x in enumerate(w):
            run += x
            if run > bound:
                break
    return n, tokens + [token] + [-1] * (T - n)
