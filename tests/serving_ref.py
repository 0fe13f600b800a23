"""Plain 64-bit implementations of the serving operators, for their tests."""
import numpy as np
import torch


def linear(q, k, v, g, S0, scale):
    """The recurrence of one request, token by token in double: q, k
    [T, HK, dk], v [T, HV, dv], g [T, HV], S0 [HV, dk, dv] (all on the CPU);
    returns (o [T, HV, dv], S)."""
    HV = v.shape[1]
    rep = HV // q.shape[1]
    q, k = (x.double().repeat_interleave(rep, 1) for x in (q, k))
    v, a, S = v.double(), g.double().exp(), S0.double().clone()
    o = torch.zeros(v.shape, dtype=torch.float64)
    for t in range(v.shape[0]):
        S = torch.where(a[t, :, None, None] > 0, a[t, :, None, None] * S, 0.0)
        S = S + k[t, :, :, None] * v[t, :, None, :]
        o[t] = scale * (q[t, :, :, None] * S).sum(1)
    return o, S


def fix40(x):
    """floor(2^40 min(max(x, 0), 1)) as Python-sized integers, NaN as 0."""
    x = np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=1.0, neginf=0.0)
    return np.floor(np.clip(x, 0.0, 1.0) * 2.0 ** 40).astype(np.int64)


def verify(p, q, tokens, u, lens):
    """(accepted, out) of p [B, K + 1, V], q [B, K, V], tokens [B, K],
    u [B, K + 1] (float64 arrays of fp32 or bf16 values) and lens [B]."""
    B, K1, V = p.shape
    accepted, out = np.zeros(B, np.int64), np.full((B, K1), -1, np.int64)
    for b in range(B):
        n = min(max(int(lens[b]), 0), K1 - 1)
        a = 0
        while a < n and 0 <= tokens[b, a] < V and \
                u[b, a] * q[b, a, tokens[b, a]] < p[b, a, tokens[b, a]]:
            out[b, a] = tokens[b, a]
            a += 1
        w = fix40(p[b, a])
        if a < n:
            w = np.maximum(w - fix40(q[b, a]), 0)
        total = int(w.sum())
        d = u[b, K1 - 1]
        r = 0 if np.isnan(d) else int(min(max(d, 0.0) * 2 ** 24, 2 ** 24 - 1))
        if total > 0:
            out[b, a] = int(np.searchsorted(np.cumsum(w), total * r >> 24, side="right"))
        accepted[b] = a
    return accepted, out


def compact(refs):
    """(map, new refs, live, [(from, to)]) of the fewest moves, ascending."""
    refs = np.asarray(refs)
    live = int((refs > 0).sum())
    moved = [s for s in range(len(refs)) if refs[s] > 0 and s >= live]
    holes = [s for s in range(live) if refs[s] <= 0]
    where = np.where(refs > 0, np.arange(len(refs)), -1)
    new = np.where(refs > 0, refs, refs * (np.arange(len(refs)) < 0))
    for a, b in zip(moved, holes):
        where[a], new[b], new[a] = b, refs[a], 0
    return where, new, live, list(zip(moved, holes))
