"""The long-cache operators in float64 (numpy) from their definitions in include/dllm.h, for the tests of the GPU calls."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
U32 = 2.0 ** -24                      # half a step of float32, relative
HALF_STEP = {"bf16": 2.0 ** -8, "f32": U32}


# ------------------------------------------------------------------------------------------------ pages

def plan_pages(page_tokens, n_pages, keep_head, length, first, table, stack, n_free):
    """Returns (table, stack, n_free, granted, bad length, bad page)."""
    table, stack = [list(r) for r in table], list(stack)
    B, NP, pt = len(table), len(table[0]), page_tokens
    bad_len = bad_page = False
    if not 0 <= n_free <= n_pages:
        bad_len, n_free = True, min(max(n_free, 0), n_pages)

    def usable(b):
        return 0 <= length[b] <= NP * pt and (first is None or first[b] >= 0)

    def needed(b, p):
        f = 0 if first is None else min(first[b], length[b])
        return p * pt < min(keep_head, length[b]) or (f // pt <= p and p * pt < length[b])
    for b in range(B):
        if not usable(b):
            bad_len = True
            continue
        for p in range(NP):
            if table[b][p] >= 0 and not needed(b, p):
                if table[b][p] < n_pages and n_free < n_pages:
                    stack[n_free] = table[b][p]
                    n_free += 1
                else:
                    bad_page = True
                table[b][p] = -1
    top, total, granted = n_free, 0, []
    for b in range(B):
        miss = [p for p in range(NP) if usable(b) and needed(b, p) and table[b][p] < 0]
        total += len(miss)
        granted.append(int(usable(b) and (not miss or total <= top)))
        for p in miss if granted[b] else []:
            n_free -= 1
            ok = 0 <= stack[n_free] < n_pages
            table[b][p] = stack[n_free] if ok else -1
            bad_page |= not ok
    return table, stack, n_free, granted, bad_len, bad_page


def slot_map(page_tokens, n_pages, start, end, table, capacity):
    """Returns (cu, slots, bad length)."""
    most, cu, slots, bad = len(table[0]) * page_tokens, [0], [], False
    for b, row in enumerate(table):
        lo, hi = (min(max(x, 0), most) for x in (start[b], end[b]))
        bad |= lo != start[b] or hi != end[b]
        for pos in range(lo, max(lo, hi)):
            page = row[pos // page_tokens]
            slots.append(page * page_tokens + pos % page_tokens if 0 <= page < n_pages else -1)
        cu.append(len(slots))
    return cu, (slots + [-1] * capacity)[:capacity], bad or len(slots) > capacity


# ------------------------------------------------------------------------------------------------ 4 bits

def encode(x):
    """x [..., 32] float64 -> codes [..., 32], scale bytes [...]."""
    x = np.asarray(x, dtype=np.float64)
    fin = np.where(np.isfinite(x), np.abs(x), 0).max(-1)
    byte = np.full(fin.shape, 7)
    while (grow := (fin > 7 * 2.0 ** (byte - 127.0)) & (byte < 252)).any():
        byte = byte + grow
    s = 2.0 ** (byte[..., None] - 127.0)
    with np.errstate(over="ignore"):
        v = np.where(np.isnan(x), 0.0, np.minimum(np.abs(x) / s, 6.0))
    d = np.abs(v[..., None] - VALUES)
    near = d == d.min(-1, keepdims=True)
    code = near.argmax(-1)
    tie = near.sum(-1) == 2
    code = np.where(tie & (code % 2 == 1), code + 1, code)          # half-way: the even one of the two
    return np.where((x < 0) & (code > 0), code + 8, code).astype(np.uint8), byte.astype(np.uint8)


def decode(code, byte):
    return np.where(code >= 8, -1.0, 1.0) * VALUES[code % 8] * 2.0 ** (byte[..., None] - 127.0)


def records(k, v):
    """k, v [32, dh] -> the record's 34 * dh bytes, and the k, v it holds."""
    dh = k.shape[1]
    ck, sk = encode(k.reshape(32, dh // 32, 32))
    cv, sv = encode(v.T)
    rec = np.zeros(34 * dh, dtype=np.uint8)
    half = rec[:16 * dh].reshape(32, dh // 2)
    half[:] = ck.reshape(32, dh)[:, ::2] | ck.reshape(32, dh)[:, 1::2] << 4
    rec[16 * dh:32 * dh].reshape(dh, 16)[:] = cv[:, ::2] | cv[:, 1::2] << 4
    ks, vs = rec[32 * dh:33 * dh].reshape(2, 4, dh // 32, 4), rec[33 * dh:].reshape(16, dh // 16)
    for s in range(32):
        ks[s // 16, s % 4, :, s // 4 % 4] = sk[s]
    for c in range(dh):
        vs[c % 16, c // 16] = sv[c]
    return rec, decode(ck, sk).reshape(32, dh), decode(cv, sv).T


# ------------------------------------------------------------------------------------------------ attention

def visible(p, n_keys, window, n_sink):
    j = np.arange(n_keys)
    return (window == 0) | (j < n_sink) | (j > p - window)


def attend(q, k, v, prefix, window, n_sink, dtype, n4=0):
    """q [nq, Hq, dh] at positions prefix .., k, v [prefix + nq, Hkv, dh].  Returns the float64 result and how far a
    correct implementation may be from it, element by element:
      scores: sums of dh products in float32, an error of (dh + 8) half steps of sum |q k| / sqrt(dh), and four half steps of the
        score itself in the scaling and the exponential; a probability's relative error is twice the largest of these
      sums over n keys: n + 64 half steps (statistics, rescaling, merging)
      probabilities enter the second product as a pair of bfloat16 (relative 2^-16) or, of keys in 4 bits, a pair of
        e4m3 (2^-4 of what is 2^-4 of it: 2^-8)
      one rounding of the output."""
    nq, hq, dh = q.shape
    out, tol = np.empty(q.shape), np.empty(q.shape)
    for h in range(hq):
        kk, vv = k[:, h // (hq // k.shape[1])], v[:, h // (hq // k.shape[1])]
        for i in range(nq):
            see = visible(prefix + i, len(kk), window, n_sink)
            ks, vs = kk[see], vv[see]
            s = ks @ q[i, h] / np.sqrt(dh)
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vs
            mag = (np.abs(ks) @ np.abs(q[i, h])).max() / np.sqrt(dh)
            rel = 2 * ((dh + 8) * mag + 4 * np.abs(s).max()) * U32 + (len(ks) + 64) * U32
            rel += 2.0 ** -8 if see[:n4].any() else (2.0 ** -16 if dtype == "bf16" else 0)
            a = rel * (w @ np.abs(vs))
            tol[i, h] = a + HALF_STEP[dtype] * (np.abs(out[i, h]) + a)
    return out, tol
