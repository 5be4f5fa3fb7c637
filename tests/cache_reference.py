"""Plain 64-bit definitions of the cache-shrinking operators, for their tests:
8-bit caches, attention weights, kept lists by score.  Written with loops over
segments and requests, apart from the library and from its timed cases."""
from __future__ import annotations

import numpy as np
import torch

BLOCK = 64


# ---------------------------------------------------------------- 8-bit format

def e4m3_values():
    """The 256 values of e4m3 (OCP): sign, 4 exponent bits of bias 7, 3 mantissa bits."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if e == 15 and m == 7:
            x = np.nan
        v[c] = -x if c & 128 else x
    return v


VALUES = e4m3_values()
_POS = VALUES[:127]  # ascending, 0 .. 448


def round_e4m3(y):
    """Codes of the nearest values (ties to the even code) of |y| <= 448, NaN for NaN."""
    y = np.asarray(y, np.float64)
    a = np.abs(np.nan_to_num(y))
    hi = np.searchsorted(_POS, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(a == _POS[hi], hi, c)
    c = c | np.where(np.signbit(y), 128, 0)
    return np.where(np.isnan(y), 127, c).astype(np.uint8)


def exponent(amax):
    e = 1
    while amax > 448 * 2.0 ** (e - 127):
        e += 1
    return e


def quantize(x, codes, exps, cu, lens=None, cu_new=None):
    """One of K and V: x[planes][src rows][d] (float64) into codes[planes][rows][d]
    and exps[planes][blocks], in place."""
    for p in range(x.shape[0]):
        for s in range(len(cu) - 1):
            beg = int(cu[s])
            n = int(lens[s]) if lens is not None else int(cu[s + 1]) - beg
            n_new = n if cu_new is None else int(cu_new[s + 1] - cu_new[s])
            src = beg if cu_new is None else int(cu_new[s])
            first = n - n_new
            for j in range(first // BLOCK, -(-n // BLOCK)):
                a, z = max(first, j * BLOCK), min(n, (j + 1) * BLOCK)
                if z <= a:
                    continue
                rows = x[p, src + a - first:src + z - first]
                slot = beg // BLOCK + s + j
                fin = np.abs(rows[np.isfinite(rows)])
                e = exponent(fin.max() if fin.size else 0.0)
                if a > j * BLOCK:
                    e_old = max(int(exps[p, slot]), 1)
                    e = max(e, e_old)
                    if e > e_old:
                        old = VALUES[codes[p, beg + j * BLOCK:beg + a]] * 2.0 ** (e_old - e)
                        codes[p, beg + j * BLOCK:beg + a] = round_e4m3(old)
                y = np.where(np.isfinite(rows), rows, np.nan)
                codes[p, beg + a:beg + z] = round_e4m3(y * 2.0 ** (127 - e))
                exps[p, slot] = e


def dequantize(codes, exps, cu, lens=None):
    """float64 values [planes][rows][d] (0 in rows of no segment)."""
    out = np.zeros(codes.shape)
    for s in range(len(cu) - 1):
        beg = int(cu[s])
        n = int(lens[s]) if lens is not None else int(cu[s + 1]) - beg
        j = np.arange(n)
        e = exps[:, beg // BLOCK + s + j // BLOCK].astype(np.float64)
        out[:, beg:beg + n] = VALUES[codes[:, beg:beg + n]] * 2.0 ** (e - 127)[..., None]
    return out


# ------------------------------------------------------------------- attention

def request_keys(w, res, ctx, b, g, layer, seg_off=None, ctx_off=None, ctx_len=None):
    """(keys [n][d], resource rows of request b and group g in order): res is
    [G][rows][d] or with seg_off a store [rows][d]."""
    rows, parts = [], []
    kept = np.asarray(w.cu_rows)
    for r in w.req_res[w.req_res_off[b]:w.req_res_off[b + 1]]:
        if not w.mask[r, layer, g]:
            continue
        n = int(kept[r + 1] - kept[r])
        a = int(seg_off[r * w.n_kv_heads + g]) if seg_off is not None else int(kept[r])
        rows.append(np.arange(a, a + n))
        parts.append(res[a:a + n] if seg_off is not None else res[g, a:a + n])
    cu = w.cu_ctx if ctx_off is None else ctx_off
    c0 = int(cu[b])
    n = int(w.ctx_lens[b])
    parts.append(ctx[g, c0:c0 + n])
    return np.concatenate(parts), np.concatenate(rows).astype(np.int64) if rows else np.zeros(0, np.int64)


def attend(w, q, rk, rv, ck, cv, layer, scale=None, seg_off=None, ctx_off=None):
    """In 64 bits: out [total_q][Hq][d], lse [Hq][total_q], and the mean distance
    of a row's values from its output under its weights, shaped as out."""
    d, R = w.head_dim, w.n_q_heads // w.n_kv_heads
    scale = scale or 1.0 / np.sqrt(d)
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.zeros((w.n_q_heads, q.shape[0]))
    for b in range(w.n_req):
        q0, tq, tc = int(w.cu_q[b]), int(w.q_lens[b]), int(w.ctx_lens[b])
        for g in range(w.n_kv_heads):
            k, rows = request_keys(w, rk, ck, b, g, layer, seg_off, ctx_off)
            v, _ = request_keys(w, rv, cv, b, g, layer, seg_off, ctx_off)
            for h in range(g * R, (g + 1) * R):
                s = q[q0:q0 + tq, h] @ k.T * scale
                for i in range(tq):
                    n = len(rows) + tc - tq + i + 1  # keys that row i sees
                    m = s[i, :n].max()
                    p = np.exp(s[i, :n] - m)
                    out[q0 + i, h] = p @ v[:n] / p.sum()
                    spread[q0 + i, h] = p @ np.abs(v[:n] - out[q0 + i, h]) / p.sum()
                    lse[h, q0 + i] = m + np.log(p.sum())
    return out, lse, spread


def attend_weights(w, q, lse, rk, ck, layer, scale=None, seg_off=None):
    """(res_w, ctx_w) in 64 bits, shaped as the keys without their last dim."""
    d, R = w.head_dim, w.n_q_heads // w.n_kv_heads
    scale = scale or 1.0 / np.sqrt(d)
    rw, cw = np.zeros(rk.shape[:-1]), np.zeros(ck.shape[:-1])
    for b in range(w.n_req):
        q0, tq, tc = int(w.cu_q[b]), int(w.q_lens[b]), int(w.ctx_lens[b])
        for g in range(w.n_kv_heads):
            k, rows = request_keys(w, rk, ck, b, g, layer, seg_off)
            vis = np.arange(len(k))[None] <= len(rows) + tc - tq + np.arange(tq)[:, None]
            total = np.zeros(len(k))
            for h in range(g * R, (g + 1) * R):
                s = q[q0:q0 + tq, h] @ k.T * scale - lse[h, q0:q0 + tq, None]
                total += np.where(vis, np.exp(np.where(vis, s, 0.0)), 0.0).sum(0)
            np.add.at(rw if seg_off is not None else rw[g], rows, total[:len(rows)])
            cw[g, int(w.cu_ctx[b]):int(w.cu_ctx[b]) + tc] += total[len(rows):]
    return rw, cw


def select(w, cu, cu_kept, keep_first, keep_last):
    """Kept lists and their weights: w float32 [planes][total]."""
    score = w.astype(np.float64).sum(0).astype(np.float32)
    kept, at = [], []
    for s in range(len(cu) - 1):
        n, k = int(cu[s + 1] - cu[s]), int(cu_kept[s + 1] - cu_kept[s])
        last = min(keep_last, k)
        first = min(keep_first, k - last)

        def rank(j):
            if j < first or j >= n - last:
                return (0, 0.0, j)
            x = score[cu[s] + j]
            return (2, 0.0, j) if np.isnan(x) else (1, -float(x), j)

        best = sorted(sorted(range(n), key=rank)[:k])
        kept += best
        at += [int(cu[s]) + j for j in best]
    return np.array(kept, np.int32), w[:, at]


def users(req_res_off, req_res, n_res):
    lists = [[] for _ in range(n_res)]
    for b in range(len(req_res_off) - 1):
        for r in req_res[req_res_off[b]:req_res_off[b + 1]]:
            lists[r].append(b)
    off = np.concatenate([[0], np.cumsum([len(x) for x in lists])])
    return off.astype(np.int32), np.array([b for x in lists for b in x], np.int32)


def host64(t):
    return t.detach().cpu().double().numpy() if isinstance(t, torch.Tensor) else np.asarray(t, np.float64)
