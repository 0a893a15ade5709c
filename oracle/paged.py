"""The paged KV cache's ops, evaluated plainly in float64 (test infrastructure only).

* Bookkeeping of a step: request by request and token by token, pages taken
  off the top of the stack of free ones as the first token of each arrives.
* Store: row by row; slots out of range are skipped.
* Attention: every row by itself over the keys it sees. Arrays hold the
  values of the dtype exactly (float64), the result is not rounded.

Attention also returns what an implementation in float32 may be off by (see
`attention`).
"""
from __future__ import annotations

import numpy as np

I32_MAX = 2 ** 31 - 1


def kv_slots(kv_len, new_len, table, free_pages, count, page, T):
    """(table, slots, pos, q_start, kv_len_out, free_out) after a step; the
    arguments are not changed."""
    table = np.array(table, dtype=np.int64)
    R, cols = table.shape
    count = min(max(int(count), 0), len(free_pages))
    slots, pos = [-1] * T, [0] * T
    q_start, out, taken = [0], [], 0
    for r in range(R):
        held = min(max(int(kv_len[r]), 0), cols * page)
        new = max(int(new_len[r]), 0)
        for col in range(-(-held // page), min(-(-(held + new) // page), cols)):
            table[r, col] = free_pages[count - 1 - taken] if taken < count else -1
            taken += 1
        for i in range(min(new, max(0, T - q_start[r]))):
            x = held + i
            col = x // page
            pid = table[r, col] if col < cols else -1
            slots[q_start[r] + i] = int(pid) * page + x % page if pid >= 0 else -1
            pos[q_start[r] + i] = x
        q_start.append(min(q_start[r] + new, I32_MAX))
        out.append(min(held + new, I32_MAX))
    return table, slots, pos, q_start, out, [max(count - taken, 0), max(taken - count, 0)]


def kv_write(k, v, slots, kc, vc):
    """The caches [n_pages, page, nk, hd] after storing rows k, v [T, nk, hd]."""
    kc, vc = kc.copy(), vc.copy()
    n, page = kc.shape[:2]
    for t, s in enumerate(slots):
        if 0 <= s < n * page:
            kc[s // page, s % page] = k[t]
            vc[s // page, s % page] = v[t]
    return kc, vc


def attention(q, kc, vc, table, kv_len, q_start, scale, window=0):
    """(out, written, spread, slack) for q [T, nq, hd] in float64.

    out [T, nq, hd]; written [T]: rows that belong to a request; spread
    [T, nq, hd] = sum_j w_j |v_j| with the softmax weights w; slack [T, nq],
    the relative error float32 arithmetic may give a weight and its sum:
    with u = 2^-24 and B_j = |scale| sum_d |q_d k_jd| a score of hd products,
    scaled, is off by at most u (hd + 3) B_j, and its distance to the maximum
    rounds by at most 2 u max|s|, taken to a power (twice, for the weight and
    for the sum it is divided by): 2 (u (hd + 3) max B + 4 u max|s|); the
    powers, the rescaling and the sums of n weights add (2 n + 200) u."""
    q, kc, vc = (np.asarray(a, dtype=np.float64) for a in (q, kc, vc))
    T, nq, hd = q.shape
    n_pages, page, nk, _ = kc.shape
    R, cols = np.shape(table)
    g, u = nq // nk, 2.0 ** -24
    out, spread = np.zeros_like(q), np.zeros_like(q)
    slack, written = np.zeros((T, nq)), np.zeros(T, dtype=bool)
    clamp = lambda x, hi: min(max(int(x), 0), hi)  # noqa: E731
    with np.errstate(all="ignore"):
        for r in range(R):
            a, b = clamp(q_start[r], T), clamp(q_start[r + 1], T)
            kv = clamp(kv_len[r], cols * page)
            at = np.arange(kv)
            pid = np.asarray(table[r], dtype=np.int64)[at // page]
            there = (pid >= 0) & (pid < n_pages)
            K = kc[np.where(there, pid, 0), at % page]
            V = vc[np.where(there, pid, 0), at % page]
            for t in range(a, b):
                written[t] = True
                p = kv - (b - t)
                see = there & (at <= p)
                if window:
                    see &= at > p - window
                if not see.any():
                    continue
                for h in range(nq):
                    Kh, Vh = K[see, h // g], V[see, h // g]
                    s = (Kh * q[t, h]).sum(-1) * scale
                    if (s == -np.inf).all():
                        continue
                    w = np.exp(s - s.max())
                    w = w / w.sum()
                    out[t, h] = (w[:, None] * Vh).sum(0)
                    spread[t, h] = (w[:, None] * np.abs(Vh)).sum(0)
                    big = (np.abs(Kh) * np.abs(q[t, h])).sum(-1).max() * abs(scale)
                    slack[t, h] = (2 * (u * (hd + 3) * big + 4 * u * np.abs(s).max())
                                   + (2 * len(s) + 200) * u)
    return out, written, spread, slack


# ---- selections ----------------------------------------------------------------------------
# Which kernels a valid call launches, from the rules alone (Python integers).
OP_KV_SLOTS, OP_KV_WRITE, OP_PAGED_ATTENTION = 12, 13, 14
KV_SLOTS, KVW_ANY, KVW_VEC = 80, 82, 83
PA_ANY, PA_ROWS, PA_TILE, PA_JOIN, PA_PAIR = 90, 91, 92, 93, 94
GRID_CAP = 1 << 20
MAX_SPLITS = 64
JOIN_WAVE = 8          # splits one wavefront joins


def _bucket(T):
    return max(0, (max(T, 1) - 1).bit_length())


def _cdiv(a, b):
    return -(-a // b)


def _k0(op, dtype, T, aligned):
    return op | dtype << 8 | _bucket(T) << 16 | int(aligned) << 24


def kv_slots_selection(T, R):
    """(key, [(variant, workgroups, work-items)]) of a kv_slots call."""
    return ((_k0(OP_KV_SLOTS, 0, T, False), 0, 0, 0, 0, 0),
            [(KV_SLOTS, min(512, _cdiv(max(T, R), 256)), 256)])


def kv_write_selection(dtype, T, nk, hd, aligned):
    """dtype 0: float32, 1: bfloat16; aligned: rows and slots at 16 bytes."""
    v = 8 if dtype else 4
    vec = aligned and hd % v == 0
    items = 2 * nk * hd // (v if vec else 1)
    return ((_k0(OP_KV_WRITE, dtype, T, aligned), 0, hd | nk << 32, 0, 0, 0),
            [(KVW_VEC if vec else KVW_ANY, min(GRID_CAP, _cdiv(T * items, 256)), 256)])


def attention_workspace(T, nq, hd, splits):
    return T * nq * splits * (hd + 2) * 4 if splits > 1 else 0


def attention_plan(dtype, T, R, nq, nk, hd, aligned, kv_max, workspace):
    """(form, splits, grids, work-items): 0 any, 1 rows, 2 tile, 3 pair; kv_max: the most
    keys a row can see."""
    v, g = (8 if dtype else 4), nq // nk
    if not aligned or hd % v or hd > 256:
        form, have, want, run, tiles, block = 0, _cdiv(T * nq, 4), 512, 256, 0, 256
    else:
        small = _cdiv(T, R) * g <= (16 if dtype else 256)
        small |= _cdiv(T * g, 16) * nk <= 64 and kv_max <= 4096
        form, m = (1, 16) if small else (2, 128)
        tiles = T * g // m + R
        have = max(_cdiv(T * g, m), min(R, T)) * nk
        want, run = (1024, 1024) if small else (256, 512 if dtype else 256)
        block = (256 if hd > 128 else 512) if small else 256
        if T % R == 0:                       # the tiles to expect: of equal chunks, or ragged ones
            fits = R * _cdiv(T // R * g, 128) * nk < (256 if R > 1 else 257)
        else:
            fits = (_cdiv(T * g, 128) + min(R, T) // 2) * nk <= 288
        if form == 2 and dtype and hd <= 128 and fits and _cdiv(T * g, 128) * nk <= 256:
            form, block = 3, 512
    s = min(want // have, _cdiv(kv_max, run))
    if form == 1 and kv_max > 512:
        s = max(s, min(256 // have, _cdiv(kv_max, 256)))
    s = max(1, min(s, MAX_SPLITS))
    while s > 1 and attention_workspace(T, nq, hd, s) > workspace:
        s -= 1
    first = tiles * nk * s if form else min(GRID_CAP, _cdiv(T * nq * s, 4))
    join = min(GRID_CAP, T * nq if s > JOIN_WAVE else _cdiv(T * nq, 4))
    return form, s, [first] + ([join] if s > 1 else []), block


def attention_selection(dtype, T, R, nq, nk, hd, aligned, kv_max, workspace):
    form, s, grids, block = attention_plan(dtype, T, R, nq, nk, hd, aligned, kv_max, workspace)
    key = (_k0(OP_PAGED_ATTENTION, dtype, T, aligned), 0, hd | nq << 16 | nk << 32,
           form << 16 | int(s > 1) << 24, 0, 0)
    launches = [((PA_ANY, PA_ROWS, PA_TILE, PA_PAIR)[form], grids[0], block)]
    if s > 1:
        launches.append((PA_JOIN, grids[1], 256))
    return key, launches
