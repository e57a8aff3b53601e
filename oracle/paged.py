"""The oracle for the paged key/value cache, in plain float64 NumPy.

TEST INFRASTRUCTURE ONLY.  Only the tests may import this module.  It shares no
code with the HIP library and imports nothing from it.

Token p of request b is row p % page_size of page table[b][p // page_size].
Batches are padded: request b has new_len[b] valid rows.  Rows that an operator
does not write keep what the output held before.
"""
from __future__ import annotations

import numpy as np

from .numerics import rms_normalize, rope


def qk_norm_rope(x, gain, eps, rope_base, past_len, new_len, out):
    """x, out [B][M][heads][D] float64: each head's row normalised (eps > 0) with gain
    (1 + gain), then rotated at position past_len[b] + row (rope_base > 0)."""
    out = np.array(out, dtype=np.float64)
    for b in range(x.shape[0]):
        m = int(new_len[b])
        y = np.asarray(x[b, :m], dtype=np.float64)
        if eps > 0:
            y = rms_normalize(y, eps) * (1.0 + (0.0 if gain is None else np.asarray(gain, dtype=np.float64)))
        if rope_base > 0 and m:
            y = rope(y, int(past_len[b]) + np.arange(m), rope_base)
        out[b, :m] = y
    return out


def paged_append(pool, table, x, past_len, new_len, rope_base=0.0):
    """The pool [n_pages][page_size][n_kv][D] float64 with rows x written (rotated where
    rope_base > 0; an 8-bit pool's values are divided by the scale afterwards, by
    whoever compares codes)."""
    pool = np.array(pool, dtype=np.float64)
    ps = pool.shape[1]
    for b in range(x.shape[0]):
        m = int(new_len[b])
        if not m:
            continue
        pos = int(past_len[b]) + np.arange(m)
        y = np.asarray(x[b, :m], dtype=np.float64)
        if rope_base > 0:
            y = rope(y, pos, rope_base)
        for t in range(m):
            pool[table[b][pos[t] // ps], pos[t] % ps] = y[t]
    return pool


def tokens_of(pool, table_row, n):
    """The first n tokens of a request: [n][n_kv][D] float64."""
    ps = pool.shape[1]
    p = np.arange(n)
    return np.asarray(pool, dtype=np.float64)[np.asarray(table_row)[p // ps], p % ps]


def visible(n_rows, kv, causal=True, window=0):
    """[n_rows][kv] truth values: row t stands at position kv - n_rows + t."""
    pos = kv - n_rows + np.arange(n_rows)[:, None]
    key = np.arange(kv)[None, :]
    ok = np.ones((n_rows, kv), dtype=bool)
    if causal:
        ok = key <= pos
        if window:
            ok &= key > pos - window
    return ok


def paged_attention(q, k_pool, v_pool, table, kv_len, new_len, out, scale=None, causal=True, window=0):
    """(o, a): the attention rows [B][M][H][D] and, for error bounds, sum_j p_j |v_j|.
    A row without a visible key is zero.  Hidden keys are taken out of the sums,
    whatever they hold."""
    B, M, H, D = q.shape
    G = H // k_pool.shape[2]
    scale = D ** -0.5 if scale is None else scale
    o = np.array(out, dtype=np.float64)
    mag = np.zeros_like(o)
    for b in range(B):
        m, n = int(new_len[b]), int(kv_len[b])
        k, v = tokens_of(k_pool, table[b], n), tokens_of(v_pool, table[b], n)
        ok = visible(m, n, causal, window)
        for t in range(m):
            at = np.flatnonzero(ok[t])
            for h in range(H):
                if not len(at):
                    o[b, t, h] = 0.0
                    continue
                s = scale * (k[at, h // G] @ np.asarray(q[b, t, h], dtype=np.float64))
                p = np.exp(s - s.max())
                p /= p.sum()
                o[b, t, h] = p @ v[at, h // G]
                mag[b, t, h] = p @ np.abs(v[at, h // G])
    return o, mag


def paged_gather(k_pool, v_pool, table, kv_len, rows):
    """[2][B][rows][n_kv * D] of one layer, zeros behind kv_len[b]."""
    B, kd = len(kv_len), k_pool.shape[2] * k_pool.shape[3]
    out = np.zeros((2, B, rows, kd))
    for b in range(B):
        n = int(kv_len[b])
        for i, pool in enumerate((k_pool, v_pool)):
            out[i, b, :n] = tokens_of(pool, table[b], n).reshape(n, kd)
    return out


def prefill_chunks(cfg, weights, x, chunks, causal):
    """K/V of one request's tokens fed in chunks: x [n, d], chunks: (length, causal) of each.
    A token sees every token of the chunks before its own, and of its own all (causal
    false) or those up to itself.  Returns [L][2][n][n_kv * d_h]."""
    from .numerics import attention, decode_stored, gelu_tanh
    L, nq, nkv, D, n = cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, x.shape[0]
    pos, allowed, at = np.arange(n), np.zeros((n, n), dtype=bool), 0
    for m, up_to in zip(chunks, causal):
        rows = slice(at, at + m)
        allowed[rows, :at + m] = True
        if up_to:
            allowed[rows] &= pos[None, :] <= pos[rows, None]
        at += m
    out, h = np.zeros((L, 2, n, nkv * D)), np.asarray(x, dtype=np.float64)

    def W(name):
        return decode_stored(weights[name]).astype(np.float64, copy=False)

    for l in range(L):
        p = f"layers.{l}."
        a = rms_normalize(h, cfg.rms_eps) * (1.0 + W(p + "attn_norm")[0])
        q, k, v = ((a @ W(p + w)).reshape(n, -1, D) for w in ("wq", "wk", "wv"))
        if cfg.rope:
            q, k = rope(q, pos, cfg.rope_base), rope(k, pos, cfg.rope_base)
        out[l, 0], out[l, 1] = k.reshape(n, nkv * D), v.reshape(n, nkv * D)
        if l + 1 == L:
            break
        h = h + attention(q, k, v, allowed).reshape(n, nq * D) @ W(p + "wo")
        m = rms_normalize(h, cfg.rms_eps) * (1.0 + W(p + "mlp_norm")[0])
        h = h + (gelu_tanh(m @ W(p + "w_gate")) * (m @ W(p + "w_up"))) @ W(p + "w_down")
    return out
