"""64-bit restatements of the verification-step operators (plain numpy / python, one loop per sequence), for the tests."""
from __future__ import annotations

import math

import numpy as np

PAGE = 128


def plan(past, new, owned, table, free, n_free, max_blocks):
    """Pages handed out one by one, as a host allocator would."""
    stack, out, got, slots, pos, missing = list(free[:n_free]), [], [], [], [], 0
    for b in range(len(past)):
        row = list(table[b][: owned[b]])
        want = -(-(past[b] + new[b]) // PAGE)
        while len(row) < want:
            if len(row) < max_blocks and stack:
                row.append(stack.pop())
            else:
                missing += want - len(row)
                break
        got.append(len(row))
        for p in range(past[b], past[b] + new[b]):
            held = row[p // PAGE] if p // PAGE < len(row) else -1
            slots.append(held * PAGE + p % PAGE if held >= 0 else -1)
            pos.append(p)
        out.append(row + [-1] * (max_blocks - len(row)))
    cu = np.concatenate([[0], np.cumsum(new)])
    return {"block_table": np.array(out), "n_owned": np.array(got), "n_free": np.array([len(stack)]), "cu_new": cu, "slot_map": np.array(slots, dtype=np.int64),
            "positions": np.array(pos, dtype=np.int64),
            "info": np.array([cu[-1], n_free - len(stack), missing, max(p + n for p, n in zip(past, new))])}


def angles(positions, hd, theta):
    return np.asarray(positions, np.float64)[:, None] * theta ** (-np.arange(0, hd, 2, dtype=np.float64) / hd)


def head_norm(x, gain, eps):
    return x if gain is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def rotate(h, positions, theta, sign=1.0):
    hd = h.shape[-1]
    a = angles(positions, hd, theta)[:, None]
    c, s = np.cos(a), sign * np.sin(a)
    lo, hi = h[..., : hd // 2], h[..., hd // 2:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def norm_rope_bwd(x, dy, gain, eps, positions, theta):
    dz = rotate(dy, positions, theta, -1.0)
    if gain is None:
        return dz, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, dh = x * r, dz * gain
    return r * (dh - xh * (dh * xh).mean(-1, keepdims=True)), (dz * xh).sum((0, 1))


def tree_attention(q, k, v, past, cu, rows, sees, scale=None, v_scale=None, v_codes=None):
    """q [T, n_q, hd]; k, v [cache rows, n_kv, hd] (values); rows[b]: cache row of every key of sequence b (-1: reads as zeros); sees[b]:
    bool [new, new].  -> out, lse, A (sum p |v|, what a relative error of the probabilities is multiplied with), Z (the largest
    sum |q k| scale of a row, what a relative error of the products is multiplied with), and with v_scale / v_codes (v being their product)
    G = max_j(p_j scale_j) sum_j |code_j|, what an error relative to a row's largest scale-weighted probability is multiplied with."""
    T, n_q, hd = q.shape
    rep = n_q // k.shape[1]
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out, lse = np.zeros((T, n_q, hd)), np.full((T, n_q), -np.inf)
    A, Z, G = np.zeros((T, n_q, hd)), np.zeros((T, n_q)), np.zeros((T, n_q, hd))
    for b in range(len(past)):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        r = np.asarray(rows[b])
        kb, vb = np.where((r >= 0)[:, None, None], k[np.maximum(r, 0)], 0.0), np.where((r >= 0)[:, None, None], v[np.maximum(r, 0)], 0.0)
        vis = np.concatenate([np.ones((n, past[b]), bool), sees[b]], 1)
        for i in range(n):
            kk, vv = kb[vis[i]], vb[vis[i]]
            if not len(kk):
                continue
            for h in range(n_q):
                x = q[cu[b] + i, h]
                z = kk[:, h // rep] @ x * scale
                m = z.max()
                p = np.exp(z - m)
                out[cu[b] + i, h] = p @ vv[:, h // rep] / p.sum()
                A[cu[b] + i, h] = p @ np.abs(vv[:, h // rep]) / p.sum()
                Z[cu[b] + i, h] = (np.abs(kk[:, h // rep]) @ np.abs(x)).max() * scale
                lse[cu[b] + i, h] = m + np.log(p.sum())
                if v_scale is not None:
                    seen = np.maximum(r, 0)[vis[i]]
                    G[cu[b] + i, h] = (p * v_scale[seen]).max() / p.sum() * np.abs(v_codes[seen, h // rep]).sum(0)
    return out, lse, A, Z, G


def token_logprobs(x, targets, temperature, top_k):
    z = x / temperature
    m = z.max(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.exp(z - m)
        l = p.sum(1, keepdims=True)
        logp = z - m - np.log(l)
        ent = -np.where(p > 0, p / l * logp, 0.0).sum(1)
        lse = (m + np.log(l))[:, 0]
    t = np.asarray(targets)
    lp = np.where(t >= 0, logp[np.arange(len(t)), np.maximum(t, 0)], 0.0)
    ids = np.argsort(-x, 1, kind="stable")[:, :top_k]
    return {"logprob": lp, "entropy": ent, "lse": lse, "top_ids": ids, "top_logprobs": np.take_along_axis(logp, ids, 1)}


def token_logprobs_bwd(x, targets, temperature, g_lp, g_h):
    z = x / temperature
    m = z.max(1, keepdims=True)
    logp = z - m - np.log(np.exp(z - m).sum(1, keepdims=True))
    p = np.exp(logp)
    h = -np.where(p > 0, p * logp, 0.0).sum(1, keepdims=True)
    t = np.asarray(targets)
    known = (t >= 0).astype(np.float64)
    one = np.zeros_like(p)
    one[np.arange(len(t)), np.maximum(t, 0)] = known
    d = g_lp[:, None] * (one - p * known[:, None])
    if g_h is not None:
        d = d - g_h[:, None] * np.where(p > 0, p * (logp + h), 0.0)
    return d / temperature
