"""The paged cache in 64 bits: positions of the compacted rows, the append with
its rotation, and attention over runs and shared prefixes, from the definitions
in ``include/stepprune.h``.  NumPy float64, row by row.
"""
import numpy as np


def compact_positions(vis_pos, img_off, text_pos, text_off, kept, layout, rows_per_image, out):
    """``out`` [axes, out_rows] with the rows of the compacted buffer filled in."""
    out = np.array(out)
    at = 0
    for b in range(len(img_off) - 1):
        if layout == "padded":
            at = b * rows_per_image
        for i in kept[b]:
            out[:, at] = vis_pos[:, img_off[b] + i]
            at += 1
        for t in range(text_off[b], text_off[b + 1]):
            out[:, at] = text_pos[:, t]
            at += 1
    return out


def rotate(x, angles, interleaved):
    """x [..., D] with its first 2 len(angles) elements turned; angles [pairs, 2] (cos, sin)."""
    y = np.array(x, np.float64)
    pairs = angles.shape[0]
    for j in range(pairs):
        p, q = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
        c, s = angles[j]
        y[..., p], y[..., q] = x[..., p] * c - x[..., q] * s, x[..., q] * c + x[..., p] * s
    return y


def append(k_cache, v_cache, q, k, v, first, counts, tables, lens, cos_sin=None, pos=None, section=None,
           interleaved=False):
    """Caches [pages, heads, page, D] and q [rows, heads, D] after the append, in 64 bits.
    first, counts: rows of every sequence; pos [axes, rows] or None: the slots."""
    k_cache, v_cache = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    q_out = np.array(q, np.float64)
    page = k_cache.shape[2]
    for s, n in enumerate(counts):
        for i in range(n):
            row, slot = first[s] + i, lens[s] - n + i
            kk, qq = np.asarray(k[row], np.float64), np.asarray(q[row], np.float64)
            if cos_sin is not None:
                axis = np.repeat(np.arange(len(section)), section)
                at = [slot if pos is None else pos[a, row] for a in axis]
                angles = np.stack([cos_sin[p, j] for j, p in enumerate(at)]).astype(np.float64)
                kk, qq = rotate(kk, angles, interleaved), rotate(qq, angles, interleaved)
            where = tables[s][slot // page], slice(None), slot % page
            k_cache[where], v_cache[where], q_out[row] = kk, v[row], qq
    return q_out, k_cache, v_cache


def run_tokens(cache, table, length):
    """The tokens of a run, [length, heads, D]."""
    page = cache.shape[2]
    out = np.zeros((length,) + (cache.shape[1], cache.shape[3]))
    for p in range(length):
        out[p] = cache[table[p // page], :, p % page]
    return out


def attend(q, k_cache, v_cache, first, counts, tables, lens, scale, prefix_tables=(), prefix_lens=(), grp_off=(),
           see_all=False):
    """(o [rows, heads, D], lse [rows, heads]) in 64 bits; rows of no sequence are NaN."""
    rows, Hq, D = q.shape
    Hk = k_cache.shape[1]
    o, lse = np.full(q.shape, np.nan), np.full((rows, Hq), np.nan)
    for s, n in enumerate(counts):
        own_k, own_v = run_tokens(k_cache, tables[s], lens[s]), run_tokens(v_cache, tables[s], lens[s])
        pre_k, pre_v = own_k[:0], own_v[:0]
        for g in range(len(prefix_lens)):
            if grp_off[g] <= s < grp_off[g + 1]:
                pre_k = run_tokens(k_cache, prefix_tables[g], prefix_lens[g])
                pre_v = run_tokens(v_cache, prefix_tables[g], prefix_lens[g])
        for i in range(n):
            seen = lens[s] if see_all else max(0, min(lens[s], lens[s] - n + i + 1))
            K, V = np.concatenate([pre_k, own_k[:seen]]), np.concatenate([pre_v, own_v[:seen]])
            for h in range(Hq):
                g = h // (Hq // Hk)
                row = first[s] + i
                if len(K) == 0:
                    o[row, h], lse[row, h] = 0.0, -np.inf
                    continue
                sc = scale * (K[:, g] @ np.asarray(q[row, h], np.float64))
                m = sc.max()
                p = np.exp(sc - m)
                o[row, h] = p @ V[:, g] / p.sum()
                lse[row, h] = m + np.log(p.sum())
    return o, lse
