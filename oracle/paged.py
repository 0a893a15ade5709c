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


def attention(q, kc, vc, table, kv_len, q_start, scale, window=0, more=0):
    """(out, written, spread, slack) for q [T, nq, hd] in float64.

    out [T, nq, hd]; written [T]: rows that belong to a request; spread
    [T, nq, hd] = sum_j w_j |v_j| with the softmax weights w; slack [T, nq],
    the relative error float32 arithmetic may give a weight and its sum:
    with u = 2^-24 and B_j = |scale| sum_d |q_d k_jd| a score of hd products,
    scaled, is off by at most u (hd + 3) B_j, and its distance to the maximum
    rounds by at most 2 u max|s|, taken to a power (twice, for the weight and
    for the sum it is divided by): 2 (u (hd + 3) max B + 4 u max|s|); the
    powers, the rescaling and the sums of n weights add (2 n + 200) u. `more`
    roundings of a score to be counted beside those."""
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
                    slack[t, h] = (2 * (u * (hd + 3) * big + (4 + more) * u * np.abs(s).max())
                                   + (2 * len(s) + 200) * u)
    return out, written, spread, slack


# ---- the cache in 8 bits ----
# Codes are held as the numbers they are (float64: whole numbers, or e4m3's values), scales
# [n_pages, page / block, nk] as float32's; what a slot holds is code * scale.
INT8, E4M3 = 0, 1
CODE_MAX = (127.0, 448.0)


def _places(r, table, kv_len, q_start, T, page, n_pages):
    """(row, position, page id or -1) of each row of request r, and its tokens' number."""
    clamp = lambda x, hi: min(max(int(x), 0), hi)  # noqa: E731
    a, b = clamp(q_start[r], T), clamp(q_start[r + 1], T)
    kv = clamp(kv_len[r], np.shape(table)[1] * page)
    out = []
    for t in range(a, b):
        p = kv - (b - t)
        pid = int(table[r][p // page]) if p >= 0 else -1
        out.append((t, p, pid if 0 <= pid < n_pages else -1))
    return out


def nearest_code(y, code):
    """The code nearest to y, ties to the even one: whole numbers, or three bits behind the
    leading one, in steps of no less than 2^-9."""
    y = np.asarray(y, dtype=np.float64)
    if code == INT8:
        return np.rint(y)
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(y))), -6.0)
    step = 2.0 ** (e - 3)
    return np.rint(y / step) * step


def scale_for(most, code):
    """The float32 scale of values up to `most`."""
    if not np.isfinite(most):
        return np.float32(np.nan)
    if code == INT8:
        s = np.float32(most) / np.float32(127)
    else:
        m, e = np.frexp(np.float64(most) / 448)      # (the power of two at or above)
        s = np.ldexp(1.0, int(e) - (m == 0.5)) if most else 0.0
    return np.float32(max(float(s), 2.0 ** -100))


def kv_write_q8(k, v, kc, vc, ks, vs, table, kv_len, q_start, code):
    """(kc, vc, ks, vs) after the call, block by block and head by head."""
    kc, vc, ks, vs = (np.array(x) for x in (kc, vc, ks, vs))
    n_pages, page, nk, _ = kc.shape
    block = page // ks.shape[1]
    for r in range(len(table)):
        blocks = {}
        for t, p, pid in _places(r, table, kv_len, q_start, len(k), page, n_pages):
            if pid >= 0:
                blocks.setdefault((pid, p % page // block), []).append((t, p % page))
        for (pid, b), rows in blocks.items():
            held = list(range(b * block, rows[0][1]))
            slots = [s for _, s in rows]
            for x, c, sc in ((k, kc, ks), (v, vc, vs)):
                for h in range(nk):
                    y = np.asarray(x[[t for t, _ in rows], h], dtype=np.float64)
                    need, was = scale_for(np.abs(y).max(), code), sc[pid, b, h]
                    now = was if held and not (need > was or np.isnan(need)) else need
                    if held and now > was:
                        z = c[pid, held, h] * np.float64(was) / np.float64(now)
                        c[pid, held, h] = nearest_code(z, code)
                    sc[pid, b, h] = now
                    if np.isnan(now):
                        c[pid, slots, h] = 0.0
                        continue
                    z = y / np.float64(now)
                    c[pid, slots, h] = nearest_code(z if code == INT8 else np.float32(z), code)
    return kc, vc, ks, vs


def values_q8(c, s):
    """What the slots of a cache hold."""
    with np.errstate(all="ignore"):
        return np.asarray(c, np.float64) * np.repeat(np.float64(s), c.shape[1] // s.shape[1], 1)[..., None]


def kv_read_q8(kc, vc, ks, vs, table, kv_len, q_start, T):
    """(k, v [T, nk, hd], which rows belong to a request)."""
    k, v = (np.zeros((T,) + kc.shape[2:]) for _ in range(2))
    written = np.zeros(T, dtype=bool)
    K, V = values_q8(kc, ks), values_q8(vc, vs)
    for r in range(len(table)):
        for t, p, pid in _places(r, table, kv_len, q_start, T, kc.shape[1], len(kc)):
            written[t] = True
            if pid >= 0:
                k[t], v[t] = K[pid, p % kc.shape[1]], V[pid, p % kc.shape[1]]
    return k, v, written


# ---- selections ----------------------------------------------------------------------------
# Which kernels a valid call launches, from the rules alone (Python integers).
OP_KV_SLOTS, OP_KV_WRITE, OP_PAGED_ATTENTION = 12, 13, 14
KV_SLOTS, KVW_ANY, KVW_VEC = 80, 82, 83
PA_ANY, PA_ROWS, PA_TILE, PA_JOIN, PA_PAIR = 90, 91, 92, 93, 94
OP_KV_WRITE_Q8, OP_KV_READ_Q8, OP_PAGED_ATTENTION_Q8 = 15, 16, 17
Q8W_ANY, Q8W_VEC, Q8R_ANY, Q8R_VEC = 100, 101, 102, 103
PA8_ANY, PA8_ROWS, PA8_TILE, PA8_PAIR, PA8_JOIN = 104, 105, 106, 107, 108
GRID_CAP = 1 << 20
MAX_SPLITS = 64
JOIN_WAVE = 8          # splits one wavefront joins
MAX_SPLITS_Q8 = 128    # of few rows over an 8-bit cache


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


def kv_rows_q8_selection(op, dtype, code, T, R, nk, hd, block, aligned):
    """kv_write_q8 or kv_read_q8; aligned: rows at 16 bytes, slots at a vector's codes."""
    v = 8 if dtype else 4
    vec = aligned and hd % v == 0
    key = [_k0(op, dtype, T, aligned), 0, hd | nk << 32, code << 32, 0, 0]
    if op == OP_KV_READ_Q8:
        return tuple(key), [(Q8R_VEC if vec else Q8R_ANY, min(GRID_CAP, _cdiv(T, 4)), 256)]
    units, parts = min(T, T // block + 2 * R), 2 * nk       # blocks that the rows can touch
    team = 1                                                # a wavefront
    if vec:
        vecs = min(_cdiv(T, R), block) * (hd // v)
        team = 0 if vecs <= 128 else 1 if vecs <= 512 else 2
        key[3] |= team << 16
    if team == 0:                                           # 16 lanes; heads one after the other
        groups = _cdiv(parts, 4)
        inner = max(1, min(groups, units * groups // 4096))
        waves = units * _cdiv(parts, 4 * inner)
    else:
        waves = units * parts * (4 if team == 2 else 1)
    return tuple(key), [(Q8W_VEC if vec else Q8W_ANY, min(GRID_CAP, _cdiv(waves, 4)), 256)]


def attention_q8_plan(dtype, T, R, nq, nk, hd, aligned, kv_max, keys_max, workspace):
    """(form, splits, grids, work-items, log2 of a tile's K heads, log2 of a step's keys)."""
    g, heads, shift = nq // nk, 0, 0
    rows, rpr, busy = T * nq, _cdiv(T, R) * g, min(R, T)
    fits = lambda s: s < 2 or attention_workspace(T, nq, hd, s) <= workspace  # noqa: E731
    if not (aligned and hd % 16 == 0 and hd <= 256):
        form, block = 0, 256
        s = min(512 // _cdiv(rows, 4), _cdiv(kv_max, 256), MAX_SPLITS)
    elif rpr <= 16 or (_cdiv(T * g, 16) * nk <= 64 and kv_max <= 4096):
        form, block = 1, 256 if hd > 128 else 512
        short = kv_max <= 1024
        if not (short and busy * nk < 1024):
            heads = max(x for x in range(3) if x == 0 or (nk % (1 << x) == 0 and rpr <= 16 >> x))
        groups, m = nk >> heads, 16 >> heads
        tiles = (T * g // m + R) * groups
        s = 1
        if not short and max(_cdiv(T * g, m), busy) * groups < 4096:
            s = min(MAX_SPLITS_Q8, (1 << 27) // (rows * (hd + 2) * 4))
        shift = (8 if hd > 128 else 9) - heads
        first = min(256, tiles * _cdiv(kv_max, 1 << shift))
        while tiles * _cdiv(keys_max, 1 << shift) >= 1 << 31:
            shift += 1
    else:
        form, block, full = 2, 256, _cdiv(T * g, 128)
        s = min(256 // (max(full, busy) * nk), _cdiv(kv_max, 512 if dtype else 256), MAX_SPLITS)
        if T % R == 0:
            few = R * _cdiv(T // R * g, 128) * nk < (256 if R > 1 else 257)
        else:
            few = (full + busy // 2) * nk <= 288
        if dtype and hd <= 128 and few and full * nk <= 256:
            form, block = 3, 512
    while not fits(s):
        s -= 1
    s = max(1, s)
    if form == 0:
        first = min(GRID_CAP, _cdiv(rows * s, 4))
    elif form > 1:
        first = (T * g // 128 + R) * nk * s
    four = rows < 512 if form == 1 else s > JOIN_WAVE
    join = min(GRID_CAP, rows if four else _cdiv(rows, 4))
    return form, s, [first] + ([join] if s > 1 else []), block, heads, shift


def attention_q8_selection(dtype, code, T, R, nq, nk, hd, aligned, kv_max, keys_max, workspace):
    form, s, grids, block, heads, _ = attention_q8_plan(dtype, T, R, nq, nk, hd, aligned, kv_max,
                                                        keys_max, workspace)
    key = (_k0(OP_PAGED_ATTENTION_Q8, dtype, T, aligned), 0, hd | nq << 16 | nk << 32,
           form << 16 | int(s > 1) << 24 | heads << 25 | code << 32, 0, 0)
    launches = [((PA8_ANY, PA8_ROWS, PA8_TILE, PA8_PAIR)[form], grids[0], block)]
    if s > 1:
        launches.append((PA8_JOIN if form == 1 else PA_JOIN, grids[1], 256))
    return key, launches
