"""Oracle 8-bit paged KV cache: number formats, block scales, the writers,
attention over it, and the block tables that give requests their pages.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A page holds [Hkv][page_size][128] bytes; 32 consecutive tokens of a head share
a scale ([Hkv][page_size / 32]).  A byte is a sign, exponent bits and mantissa
bits (e4m3: 4 and 3, bias 7, no infinity, NaN = all ones; e5m2: 5 and 2, bias
15, infinity and NaN as in IEEE formats).  Appending values x to a block with o
tokens takes scale = max(old, need) (need alone if o = 0), need the smallest
power of two in [2^-60, 2^60] with max finite |x| <= largest * need; bytes are
x / scale to the nearest (ties to even), saturated; where the scale grows the
old bytes' values are divided by the ratio and rounded again.
"""
import numpy as np

from . import status as st

BLOCK = 32
E4M3, E5M2 = 0, 1
# exponent bias, mantissa bits, largest value
FORMATS = {E4M3: (7, 3, 448.0), E5M2: (15, 2, 57344.0)}


def decode8(code, fmt):
    """Bytes to float64."""
    bias, man, _ = FORMATS[fmt]
    c = np.asarray(code, np.uint8).astype(np.int64)
    sign = np.where(c & 0x80, -1.0, 1.0)
    e = (c & 0x7F) >> man
    m = c & ((1 << man) - 1)
    x = np.where(e == 0, np.ldexp(m.astype(np.float64), 1 - bias - man),
                 np.ldexp((m + (1 << man)).astype(np.float64), (e - bias - man).astype(np.int32)))
    if fmt == E4M3:
        x = np.where((c & 0x7F) == 0x7F, np.nan, x)
    else:
        x = np.where(e == 31, np.where(m == 0, np.inf, np.nan), x)
    return sign * x


def encode8(x, fmt):
    """float64 to bytes: the nearest value (ties to the even mantissa), magnitudes beyond
    the largest saturated, NaN to a NaN of either sign."""
    _, _, top = FORMATS[fmt]
    x = np.asarray(x, np.float64)
    last = 0x7E if fmt == E4M3 else 0x7B
    grid = decode8(np.arange(last + 1, dtype=np.uint8), fmt)       # increasing magnitudes
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), top)
    hi = np.minimum(np.searchsorted(grid, a, side="left"), last)   # grid[hi] >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - grid[lo], grid[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    pick = np.where(grid[hi] == a, hi, pick)
    out = pick.astype(np.uint8) | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), out).astype(np.uint8)


def bf16_to_f64(bits):
    b = np.asarray(bits, np.uint16).astype(np.uint32) << 16
    return b.view(np.float32).astype(np.float64)


def need_scale(x, fmt):
    """The smallest power of two in [2^-60, 2^60] that brings the finite values of x into
    the format's range."""
    _, _, top = FORMATS[fmt]
    fin = np.abs(x[np.isfinite(x)])
    amax = float(fin.max()) if fin.size else 0.0
    s = 2.0 ** -60
    while amax > top * s and s < 2.0 ** 60:
        s *= 2.0
    return s


def append_rows(pages, scale, fmt, page, off, x):
    """Append rows x (float64 [n, Hkv, 128]) at token `off` of a page, within one block, in
    place (one tensor)."""
    n, b, o = x.shape[0], off // BLOCK, off % BLOCK
    assert o + n <= BLOCK
    for h in range(pages.shape[1]):
        need = need_scale(x[:, h], fmt)
        old = float(scale[page, h, b])
        new = max(old, need) if o > 0 else need
        if o > 0 and new != old:
            at = pages[page, h, off - o:off]
            pages[page, h, off - o:off] = encode8(decode8(at, fmt) * (old / new), fmt)
        pages[page, h, off:off + n] = encode8(x[:, h] / new, fmt)
        scale[page, h, b] = new


def store_kv(k, v, slot_map, fmt, k_pages, v_pages, k_scale, v_scale):
    """Rows (bf16 bits [T, Hkv, 128]) to the slots of a slot map, run by run; returns
    (k_pages, v_pages, k_scale, v_scale, status)."""
    num_pages, _, ps, _ = k_pages.shape
    cache = [a.copy() for a in (k_pages, v_pages, k_scale, v_scale)]
    status, i, T = 0, 0, len(slot_map)
    while i < T:
        s = int(slot_map[i])
        if s < 0 or s >= num_pages * ps:
            if s >= 0:
                status |= st.BAD_OFFSETS
            i += 1
            continue
        n = 1
        while i + n < T and int(slot_map[i + n]) == s + n and (s + n) % BLOCK != 0:
            n += 1
        for t, x in ((0, k), (1, v)):
            append_rows(cache[t], cache[2 + t], fmt, s // ps, s % ps, bf16_to_f64(x[i:i + n]))
        i += n
    return (*cache, status)


def commit_kv_q8(q_offsets, accept_len, accept_slots, k_new, v_new, fmt, k_pages, v_pages, k_scale,
                 v_scale, block_table, prefix_len):
    """The 8-bit form of commit_kv: returns (k_pages, v_pages, k_scale, v_scale, new_len,
    status)."""
    num_pages, _, ps, _ = k_pages.shape
    cache = [a.copy() for a in (k_pages, v_pages, k_scale, v_scale)]
    new_len = np.asarray(prefix_len, np.int32).copy()
    status = 0
    for r in range(len(q_offsets) - 1):
        q0, q1 = int(q_offsets[r]), int(q_offsets[r + 1])
        if q1 <= q0:
            continue
        slots = [q0] + [int(x) for x in accept_slots[r, :int(accept_len[r])]]
        P = int(prefix_len[r])
        dest = []
        for p in range(P, P + len(slots)):
            e = p // ps
            page = int(block_table[r, e]) if e < block_table.shape[1] else -1
            dest.append(page * ps + p % ps if 0 <= page < num_pages else -1)
        if min(dest) < 0 or P + len(slots) >= 1 << 31 or not all(0 <= s < k_new.shape[0] for s in slots):
            status |= st.BAD_OFFSETS
            continue
        *cache, _ = store_kv(k_new[slots], v_new[slots], dest, fmt, *cache)
        new_len[r] = P + len(slots)
    return (*cache, new_len, status)


def cached_rows(pages, scale, fmt, block_table, r, length, head):
    """Values (float64 [length, 128]) of a head of request r's first tokens, or None if a page
    is missing."""
    num_pages, _, ps, _ = pages.shape
    out = np.zeros((length, pages.shape[3]))
    for p0 in range(0, length, ps):
        e = p0 // ps
        page = int(block_table[r, e]) if e < block_table.shape[1] else -1
        if page < 0 or page >= num_pages:
            return None
        n = min(ps, length - p0)
        f = np.repeat(scale[page, head].astype(np.float64), BLOCK)[:n]
        out[p0:p0 + n] = decode8(pages[page, head, :n], fmt) * f[:, None]
    return out


def tree_verify_attn_paged_q8(q, k_new, v_new, fmt, k_pages, v_pages, k_scale, v_scale, block_table,
                              prefix_len, q_offsets, tree_mask, hq, hkv, sm_scale):
    """Verification attention over the 8-bit cache in float64.  Returns a dict: out [Nq, Hq,
    128], lse [Nq, Hq], status, and what bounds a computation's error: dev (the mean absolute
    deviation of the values that a row weighs, per dim), vmax (their largest magnitude) and
    zabs (sm_scale times the largest sum |q_i k_i| of a visible key).  Skipped requests'
    rows stay NaN."""
    G, scale = hq // hkv, float(np.float32(sm_scale))
    nq = int(max(q_offsets))
    out = np.full((nq, hq, q.shape[2]), np.nan)
    dev, vmax = np.zeros_like(out), np.zeros((nq, hq))
    lse, zabs = np.full((nq, hq), np.nan), np.zeros((nq, hq))
    status = 0
    for r in range(len(q_offsets) - 1):
        q0, q1, P = int(q_offsets[r]), int(q_offsets[r + 1]), int(prefix_len[r])
        n = q1 - q0
        if P < 0 or n < 0 or q0 < 0 or q1 > q.shape[0]:
            status |= st.BAD_OFFSETS
            continue
        see = np.ones((n, P + n), bool)
        for s in range(n):
            for j in range(n):
                w = j >> 5
                see[s, P + j] = w < tree_mask.shape[1] and (int(tree_mask[q0 + s, w]) >> (j & 31)) & 1
        for g in range(hkv):
            K, V = (cached_rows(c, f, fmt, block_table, r, P, g)
                    for c, f in ((k_pages, k_scale), (v_pages, v_scale)))
            if K is None:
                status |= st.BAD_OFFSETS
                break
            if n == 0:
                continue
            K = np.concatenate([K, bf16_to_f64(k_new[q0:q1, g])])
            V = np.concatenate([V, bf16_to_f64(v_new[q0:q1, g])])
            for h in range(g * G, (g + 1) * G):
                Q = bf16_to_f64(q[q0:q1, h])
                z = np.where(see, scale * (Q @ K.T), -np.inf)
                za = np.where(see, scale * (np.abs(Q) @ np.abs(K).T), 0.0)
                for s in range(n):
                    vis = see[s]
                    if not vis.any():
                        out[q0 + s, h], lse[q0 + s, h] = 0.0, -np.inf
                        continue
                    m = z[s].max()
                    w = np.exp(z[s][vis] - m)
                    o = (w @ V[vis]) / w.sum()
                    out[q0 + s, h] = o
                    lse[q0 + s, h] = m + np.log(w.sum())
                    dev[q0 + s, h] = (w @ np.abs(V[vis] - o)) / w.sum()
                    vmax[q0 + s, h] = np.abs(V[vis]).max()
                    zabs[q0 + s, h] = za[s].max()
    return dict(out=out, lse=lse, status=status, dev=dev, vmax=vmax, zabs=zabs)


def build_block_tables(want_len, page_size, block_table, num_held, free_pages, num_free,
                       row_offsets=None, row_start=None, max_rows=0):
    """Give and take pages request by request (see the library's header): returns
    dict(block_table, num_held, free_pages, num_free, slot_map, status)."""
    bt, held = np.array(block_table), np.array(num_held)
    R, most = bt.shape
    stack = [int(x) for x in free_pages]
    max_free, top, status = len(stack), int(num_free), 0
    need = np.array([-(-int(x) // page_size) for x in want_len])
    ok = [0 <= int(held[r]) <= most and int(want_len[r]) >= 0 and need[r] <= most for r in range(R)]
    if not all(ok):
        status |= st.BAD_OFFSETS
    gives = sum(max(0, int(held[r]) - int(need[r])) for r in range(R) if ok[r])
    usable = 0 <= top <= max_free and top + gives <= max_free
    if not usable:
        status |= st.BAD_OFFSETS
        if any(ok[r] and need[r] > held[r] for r in range(R)):
            status |= st.NO_PAGES
    else:
        for r in range(R):
            if ok[r] and need[r] < held[r]:
                for j in range(int(need[r]), int(held[r])):
                    stack[top] = int(bt[r, j])
                    top += 1
                held[r] = need[r]
        stopped = False
        for r in range(R):
            if ok[r] and need[r] > held[r]:
                take = int(need[r] - held[r])
                if stopped or take > top:
                    stopped = True
                    status |= st.NO_PAGES
                    continue
                for j in range(int(held[r]), int(need[r])):
                    top -= 1
                    bt[r, j] = stack[top]
                held[r] = need[r]
    slots = np.full(max_rows, -1, np.int64)
    if row_offsets is not None and (min(row_offsets) < 0 or max(row_offsets) > max_rows
                                    or any(x > y for x, y in zip(row_offsets, row_offsets[1:]))):
        status |= st.BAD_OFFSETS
    elif row_offsets is not None:
        for r in range(R):
            have = int(held[r]) if 0 <= int(held[r]) <= most else 0
            for i in range(int(row_offsets[r]), min(int(row_offsets[r + 1]), max_rows)):
                p = int(row_start[r]) + i - int(row_offsets[r])
                page = int(bt[r, p // page_size]) if 0 <= p and p // page_size < have else -1
                if page < 0:
                    status |= st.NO_PAGES
                else:
                    slots[i] = page * page_size + p % page_size
    return dict(block_table=bt, num_held=held, free_pages=np.array(stack, np.int32), num_free=top,
                slot_map=slots, status=status)
