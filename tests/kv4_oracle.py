"""The paged 4-bit KV cache from its definition, in 64 bits on the CPU: codes and scales, the pool's bytes, slots, attention.
Nothing here uses the library."""
import math

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
MIN_EXP, MAX_EXP = -100, 125


def exponent(amax):
    """The smallest e with amax <= 6 * 2^e, by trying them."""
    if amax == 0:
        return 0
    e = MIN_EXP
    while e < MAX_EXP and amax > math.ldexp(6.0, e):
        e += 1
    return e


def encode_block(x):
    """(codes [32], scale byte) of 32 numbers."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    e = exponent(np.abs(x).max())
    codes = np.zeros(32, np.uint8)
    for i, v in enumerate(x):
        d = np.abs(math.ldexp(abs(v), -e) - MAGNITUDES)
        best = np.flatnonzero(d == d.min())
        codes[i] = next((c for c in best if c % 2 == 0), best[0]) | (8 if np.signbit(v) else 0)
    return codes, e + 127


def encode(x):
    """Codes [..., D] and scale bytes [..., D / 32]: encode_block over an array, the same steps for all blocks at once."""
    x = np.asarray(x, np.float64)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    fine = np.isfinite(y).all(-1)
    z = np.where(fine[..., None], y, 0.0)
    amax = np.abs(z).max(-1)
    e = np.full(amax.shape, MIN_EXP)
    for step in range(MIN_EXP, MAX_EXP):
        e = np.where((e == step) & (amax > math.ldexp(6.0, step)), step + 1, e)
    e = np.where(amax == 0, 0, e)
    d = np.abs(np.abs(np.ldexp(z, -e[..., None]))[..., None] - MAGNITUDES[[0, 2, 4, 6, 1, 3, 5, 7]])
    codes = np.array([0, 2, 4, 6, 1, 3, 5, 7])[d.argmin(-1)] + 8 * np.signbit(z)
    return codes.reshape(x.shape).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    x = VALUES[codes].reshape(*scales.shape, 32)
    with np.errstate(invalid="ignore"):
        x = np.ldexp(x, scales.astype(np.int64)[..., None] - 127)
    return np.where(scales[..., None] == 255, np.nan, x).reshape(codes.shape)


def put(pool, slots, k, v):
    """Writes rows [N, Hkv, D] into their slots of a pool [pages][Hkv][page / 16][17 D], byte by byte."""
    pages, _hkv, records, size = pool.shape
    d, page = size // 17, records * 16
    for which, x in enumerate((k, v)):
        codes, scales = encode(x)
        for n, slot in enumerate(slots):
            if not 0 <= slot < pages * page:
                continue
            p, r, t = slot // page, slot % page // 16, slot % 16
            for b in range(d // 32):
                at = which * 8 * d + (b * 16 + t) * 16
                pool[p, :, r, at:at + 16] = codes[n, :, b * 32:b * 32 + 32:2] + 16 * codes[n, :, b * 32 + 1:b * 32 + 32:2]
                pool[p, :, r, 16 * d + (b * 16 + t) * 2 + which] = scales[n, :, b]
    return pool


def get(pool, slots):
    """(K, V) [N, Hkv, D] in 64 bits of the tokens in the given slots (all inside the pool)."""
    _pages, hkv, records, size = pool.shape
    d, page, slots = size // 17, records * 16, np.asarray(slots, np.int64)
    rec = pool[slots // page, :, slots % page // 16]  # [N, Hkv, 17 D]
    t, out = slots % 16, []
    for which in range(2):
        codes = np.zeros((len(slots), hkv, d), np.uint8)
        scales = np.zeros((len(slots), hkv, d // 32), np.uint8)
        for b in range(d // 32):
            for j in range(16):
                byte = np.take_along_axis(rec, (which * 8 * d + (b * 16 + t) * 16 + j)[:, None, None].repeat(hkv, 1), 2)[..., 0]
                codes[:, :, b * 32 + 2 * j], codes[:, :, b * 32 + 2 * j + 1] = byte & 15, byte >> 4
            scales[:, :, b] = np.take_along_axis(rec, (16 * d + (b * 16 + t) * 2 + which)[:, None, None].repeat(hkv, 1), 2)[..., 0]
        out.append(values(codes, scales))
    return out


def slots(table, free, num_free, seq_len, new_len, num_rows, page, num_pages, pos_offset=None):
    """What pevlm_cache_slots leaves behind, request by request and token by token."""
    table = np.array(table)
    n = len(seq_len)
    count = min(max(num_free, 0), len(free))
    out = dict(seq_len_out=np.array(seq_len, np.int64), row_start=np.zeros(n, np.int64), row_len=np.zeros(n, np.int64),
               slot_map=np.full(num_rows, -1, np.int64), pos_ids=np.zeros(num_rows, np.int64), table=table)
    rows = wanted = taken = 0
    for s in range(n):
        held, more = max(seq_len[s], 0), max(new_len[s], 0)
        out["row_start"][s] = min(rows, 2 ** 31 - 1)
        fits = held + more <= table.shape[1] * page and rows + more <= num_rows
        have, need = -(-held // page), 0
        if fits:
            need = -(-(held + more) // page) - have
        wanted += need
        if fits and (need == 0 or wanted <= count):
            for c in range(need):
                table[s, have + c] = free[count - 1 - (wanted - need + c)]
            taken += need
            out["row_len"][s], out["seq_len_out"][s] = more, held + more
            for i in range(more):
                p = held + i
                if 0 <= table[s, p // page] < num_pages:
                    out["slot_map"][rows + i] = table[s, p // page] * page + p % page
                out["pos_ids"][rows + i] = p + (pos_offset[s] if pos_offset is not None else 0)
        rows += more
    out["num_free_out"] = np.array([count - taken])
    out["pos_ids"] = np.stack([out["pos_ids"]] * 3)
    return out


def attention(q, pool, table, kv_of_q, row_start, row_len, seq_len, sink_len=None, window=None, scale=None):
    """dict(out, lse, spread, mass): per row and head, from the formula; NaN in out and lse for rows of no request.  `spread`:
    scale * sum |q k| at its largest over the keys seen, `mass`: sum of weight * |v| per element, what rounding errors go by."""
    num_rows, hq, d = q.shape
    pages, _hkv, records, _size = pool.shape
    page, width = records * 16, table.shape[1] * records * 16
    scale = 1 / math.sqrt(d) if scale is None else scale
    r = dict(out=np.full((num_rows, hq, d), np.nan), lse=np.full((num_rows, hq), np.nan), spread=np.zeros((num_rows, hq)),
             mass=np.zeros((num_rows, hq, d)), rows=np.zeros(num_rows, bool), keys=np.zeros(num_rows, np.int64))
    for s in range(len(seq_len)):
        first, n = int(row_start[s]), int(row_len[s])
        if n <= 0 or first < 0 or first + n > num_rows:
            continue
        held = min(max(int(seq_len[s]), 0), width)
        j = np.arange(held)
        ok = (table[s, j // page] >= 0) & (table[s, j // page] < pages) if held else np.zeros(0, bool)
        k, v = get(pool, np.where(ok, table[s, j // page].astype(np.int64) * page + j % page, 0)) if held else (np.zeros((0, _hkv, d)),) * 2
        for i in range(n):
            p = held - n + i
            seen = ok & (j <= p)
            if window is not None and window[s] >= 0:
                seen &= (p - j < window[s]) | (j < (sink_len[s] if sink_len is not None else 0))
            row = first + i
            r["rows"][row], r["keys"][row] = True, seen.sum()
            if not seen.any():
                r["out"][row], r["lse"][row] = 0, -np.inf
                continue
            of = {g: (k[seen, g], v[seen, g]) for g in set(kv_of_q)}
            for h in range(hq):
                kk, vv = of[kv_of_q[h]]
                x = kk @ q[row, h].astype(np.float64) * scale
                top = x.max()
                w = np.exp(x - top)
                r["lse"][row, h] = top + np.log(w.sum())
                r["out"][row, h] = (w / w.sum()) @ vv
                r["spread"][row, h] = (np.abs(kk) @ np.abs(q[row, h].astype(np.float64))).max() * scale
                r["mass"][row, h] = (w / w.sum()) @ np.abs(vv)
    return r
