"""Oracle rotary positions and latent attention: the rotation and its tables of frequencies,
the latent paged cache's writers, and the tree attention over it, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A token's row has 576 values: 512 normalised ones (c), which every head uses as key and
as value, then 64 rotated ones, which only the scores see.  Query head h of slot s:
z_j = sm_scale * <q[s, h], row_j>, out = softmax(z) c.
"""
import numpy as np

from . import status as st
from .kvq8 import bf16_to_f64

LATENT, ROPE = 512, 64
HALF, INTERLEAVED = 0, 1


def frequencies(rot_dim, base, scaling="plain", factor=1.0, original_len=0.0, low_turns=1.0, high_turns=32.0):
    """(inverse frequencies float64 [rot_dim / 2], factor on cosines and sines)."""
    i = np.arange(rot_dim // 2)
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = np.array([base ** (-2.0 * k / rot_dim) for k in i])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "smooth":
        out = []
        for x in f:
            turns = original_len * x / (2 * np.pi)
            if turns <= low_turns:
                out.append(x / factor)
            elif turns >= high_turns:
                out.append(x)
            else:
                s = (turns - low_turns) / (high_turns - low_turns)
                out.append(s * x + (1 - s) * x / factor)
        return np.array(out), 1.0
    if scaling == "bands":
        # the (fractional) pair whose wave turns n times within original_len
        pair = lambda n: rot_dim / 2 * np.log(original_len / (2 * np.pi * n)) / np.log(base)  # noqa: E731
        lo, hi = max(np.floor(pair(high_turns)), 0), min(np.ceil(pair(low_turns)), rot_dim - 1)
        ramp = np.array([0.0 if k <= lo else 1.0 if k >= hi else (k - lo) / (hi - lo) for k in i])
        return f * (1 - ramp) + f / factor * ramp, 0.1 * np.log(factor) + 1.0
    return f, 1.0


def rotate(x, positions, inv_freq, scale, layout):
    """x float64 [rows, ..., rot] turned by its rows' positions."""
    out = np.array(x, np.float64)
    half = out.shape[-1] // 2
    for i in range(half):
        ia, ib = (2 * i, 2 * i + 1) if layout == INTERLEAVED else (i, i + half)
        t = np.asarray(positions, np.float64) * float(inv_freq[i])
        t = t.reshape((-1,) + (1,) * (out.ndim - 2))
        a, b = np.array(x[..., ia], np.float64), np.array(x[..., ib], np.float64)
        out[..., ia] = scale * (a * np.cos(t) - b * np.sin(t))
        out[..., ib] = scale * (b * np.cos(t) + a * np.sin(t))
    return out


def latent_rows(kv, weight, eps, positions, inv_freq, scale, layout):
    """The rows (float64) that kv (bf16 bits [T, 576]) becomes."""
    x = bf16_to_f64(kv[:, :LATENT + ROPE])
    out = x.copy()
    if weight is not None:
        for t in range(len(x)):
            c = x[t, :LATENT]
            out[t, :LATENT] = c / np.sqrt((c * c).mean() + float(np.float32(eps))) * bf16_to_f64(weight)
    if inv_freq is not None:
        out[:, LATENT:] = rotate(x[:, LATENT:], positions, inv_freq, scale, layout)
    return out


def slots_status(slot_map, slots):
    """(rows that go into the cache, status) of a slot map."""
    s = np.asarray(slot_map)
    return (s >= 0) & (s < slots), st.BAD_OFFSETS if (s >= slots).any() else 0


def commit_latent(q_offsets, accept_len, accept_slots, latent_new, pages, block_table, prefix_len):
    """The accepted rows appended: (pages, new_len, status)."""
    num_pages, ps, _ = pages.shape
    pages, new_len, status = pages.copy(), np.array(prefix_len, np.int32), 0
    cap, depth = latent_new.shape[0], accept_slots.shape[1]
    for r in range(len(q_offsets) - 1):
        q0, q1, n = int(q_offsets[r]), int(q_offsets[r + 1]), int(accept_len[r])
        if q1 <= q0:
            continue
        P = int(prefix_len[r])
        if q0 < 0 or q1 > cap or not 0 <= n <= depth or P < 0 or P + 1 + n >= 1 << 31:
            status |= st.BAD_OFFSETS
            continue
        slots = [q0] + [int(x) for x in accept_slots[r, :n]]
        where = []
        for p in range(P, P + 1 + n):
            e = p // ps
            page = int(block_table[r, e]) if e < block_table.shape[1] else -1
            where.append((page, p % ps) if 0 <= page < num_pages else None)
        if None in where or not all(0 <= s < cap for s in slots):
            status |= st.BAD_OFFSETS
            continue
        for s, (page, at) in zip(slots, where):
            pages[page, at] = latent_new[s]
        new_len[r] = P + 1 + n
    return pages, new_len, status


def cached_rows(pages, block_table, r, length):
    """float64 [length, 576] of request r's first tokens, or None if a page is missing."""
    num_pages, ps, row = pages.shape
    if length < 0 or length > block_table.shape[1] * ps:
        return None
    out = np.zeros((length, row))
    for p0 in range(0, length, ps):
        page = int(block_table[r, p0 // ps])
        if page < 0 or page >= num_pages:
            return None
        n = min(ps, length - p0)
        out[p0:p0 + n] = bf16_to_f64(pages[page, :n])
    return out


def tree_verify_attn_latent(q, latent_new, pages, block_table, prefix_len, q_offsets, tree_mask, hq, sm_scale):
    """Returns a dict: out [Nq, Hq, 512], lse [Nq, Hq], status, and what bounds a
    computation's error (as kvq8.tree_verify_attn_paged_q8): dev, vmax, zabs.  Skipped
    requests' rows stay NaN."""
    scale = float(np.float32(sm_scale))
    nq = max(int(max(q_offsets)), 0)
    out = np.full((nq, hq, LATENT), np.nan)
    dev, vmax = np.zeros_like(out), np.zeros((nq, hq))
    lse, zabs = np.full((nq, hq), np.nan), np.zeros((nq, hq))
    status = 0
    for r in range(len(q_offsets) - 1):
        q0, q1, P = int(q_offsets[r]), int(q_offsets[r + 1]), int(prefix_len[r])
        n = q1 - q0
        if n < 0 or q0 < 0 or q1 > q.shape[0] or P < 0 or P > block_table.shape[1] * pages.shape[1]:
            status |= st.BAD_OFFSETS
            continue
        if n == 0:
            continue
        cached = cached_rows(pages, block_table, r, P)
        if cached is None:
            status |= st.BAD_OFFSETS
            continue
        K = np.concatenate([cached, bf16_to_f64(latent_new[q0:q1])])
        for s in range(n):
            vis = [True] * P + [j >> 5 < tree_mask.shape[1] and bool((int(tree_mask[q0 + s, j >> 5]) >> (j & 31)) & 1)
                                for j in range(n)]
            V = K[np.array(vis, bool)]
            for h in range(hq):
                if not len(V):
                    out[q0 + s, h], lse[q0 + s, h] = 0.0, -np.inf
                    continue
                Q = bf16_to_f64(q[q0 + s, h])
                z = scale * (V @ Q)
                w = np.exp(z - z.max())
                o = w @ V[:, :LATENT] / w.sum()
                out[q0 + s, h], lse[q0 + s, h] = o, z.max() + np.log(w.sum())
                dev[q0 + s, h] = w @ np.abs(V[:, :LATENT] - o) / w.sum()
                vmax[q0 + s, h] = np.abs(V[:, :LATENT]).max()
                zabs[q0 + s, h] = scale * (np.abs(V) @ np.abs(Q)).max()
    return dict(out=out, lse=lse, status=status, dev=dev, vmax=vmax, zabs=zabs)
