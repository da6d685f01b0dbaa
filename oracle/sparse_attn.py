"""CPU oracle for attention over chosen key blocks.  TEST INFRASTRUCTURE ONLY.

fp64 numpy, one query at a time's worth of definition: the keys are cut into numbered blocks (every cache frame on its
own, then the chunk), a query attends to the concatenation of the blocks its list names (a block named twice counts
twice; an entry outside the range names none), an empty list gives O = 0 and LSE = -inf.  Shares nothing with the CUDA path.
"""
from __future__ import annotations

import numpy as np

QUERY_BLOCK = 128


def key_blocks(held_frames: int, tokens_per_frame: int, n_kc: int, block: int):
    """List of (first, end) token ranges in [context frames in logical order; chunk]."""
    out = []
    for f in range(held_frames):
        for t in range(0, tokens_per_frame, block):
            out.append((f * tokens_per_frame + t, f * tokens_per_frame + min(t + block, tokens_per_frame)))
    ctx = held_frames * tokens_per_frame
    for t in range(0, n_kc, block):
        out.append((ctx + t, ctx + min(t + block, n_kc)))
    return out


def block_means(k, ranges):
    """k [tokens, D] -> [blocks, D]."""
    return np.stack([k[a:b].mean(0) for a, b in ranges]) if ranges else np.zeros((0, k.shape[1]))


def select(q, k, ranges, n_select, kept=()):
    """q [n_q, D], k [tokens, D] (float64) of one head: lists [query blocks, n_select], -1 padded, ascending."""
    means = block_means(k, ranges).astype(np.float32).astype(np.float64)
    out = []
    for i in range(0, q.shape[0], QUERY_BLOCK):
        qm = q[i:i + QUERY_BLOCK].mean(0).astype(np.float32).astype(np.float64)
        s = means @ qm
        plain = [j for j in range(len(ranges)) if j not in kept]
        rank = sorted(kept) + sorted(plain, key=lambda j: (bool(np.isnan(s[j])), 0.0 if np.isnan(s[j]) else -s[j], j))
        chosen = sorted(rank[:n_select])
        out.append(chosen + [-1] * (n_select - len(chosen)))
    return np.array(out, np.int64)


def _keys_of(row, ranges):
    parts = [np.arange(*ranges[j]) for j in row if 0 <= j < len(ranges)]
    return np.concatenate(parts) if parts else np.zeros(0, np.int64)


def attend(q, k, v, blocks, ranges, scale, d_o=None, n_ctx_tokens=0):
    """One head: q [n_q, D], k, v [tokens, D], blocks [query blocks, n]; returns (O, LSE) or, with d_o, (O, LSE, dQ, dK, dV)
    with dK, dV of the tokens from n_ctx_tokens on."""
    n_q, D = q.shape
    o, lse, dq = np.zeros((n_q, D)), np.full(n_q, -np.inf), np.zeros((n_q, D))
    dk, dv = np.zeros_like(k), np.zeros_like(v)
    for qb in range(blocks.shape[0]):
        rows = slice(qb * QUERY_BLOCK, min(n_q, (qb + 1) * QUERY_BLOCK))
        at = _keys_of(blocks[qb], ranges)
        if at.size == 0:
            continue
        s = scale * (q[rows] @ k[at].T)
        m = s.max(1, keepdims=True)
        e = np.exp(s - m)
        p = e / e.sum(1, keepdims=True)
        lse[rows] = (m + np.log(e.sum(1, keepdims=True)))[:, 0]
        o[rows] = p @ v[at]
        if d_o is not None:
            g = d_o[rows]
            ds = scale * p * (g @ v[at].T - (g * o[rows]).sum(1, keepdims=True))
            dq[rows] = ds @ k[at]
            np.add.at(dk, at, ds.T @ q[rows])
            np.add.at(dv, at, p.T @ g)
    if d_o is None:
        return o, lse
    return o, lse, dq, dk[n_ctx_tokens:], dv[n_ctx_tokens:]
