"""The paged key-value cache in plain numpy, 64 bits, token by token: what the GPU tests compare with."""
import numpy as np


def tokens_of(table_row, n, P, n_pages):
    """[(position, page, row)] of the first n positions that have a page."""
    out = []
    for j in range(min(n, len(table_row) * P)):
        page = int(table_row[j // P])
        if 0 <= page < n_pages:
            out.append((j, page, j % P))
    return out


def attend(q, k, v, sizes, table, lengths, scale, enhance):
    """q [S, Hq, D], k, v [n_pages, H, P, D], sizes [n_pages, P] or None, all float64 / int.  Returns (out, bulk, steep, live):
    out = sum_j a_j (v_j + log s_j), bulk = sum_j a_j |v_j + log s_j| (what a relative error of the weights or a rounding of a
    partial sum acts on), steep = the largest scale * sum_d |q_d k_jd| (what a relative error of the products of a logit acts on)
    per sequence and head, live = tokens per sequence."""
    S, Hq, D = q.shape
    n_pages, H, P, _ = k.shape
    G = Hq // H
    out, bulk, steep, live = np.zeros((S, Hq, D)), np.zeros((S, Hq, D)), np.zeros((S, Hq, 1)), np.zeros(S, int)
    for s in range(S):
        at = [(p, r) for _, p, r in tokens_of(table[s], int(lengths[s]), P, n_pages) if sizes is None or sizes[p, r] >= 1]
        live[s] = len(at)
        if not at:
            continue
        p, r = np.array([a for a, _ in at]), np.array([b for _, b in at])
        ls = np.log(sizes[p, r].astype(np.float64))[:, None] if enhance else 0.0
        for h in range(Hq):
            kk, vv = k[p, h // G, r], v[p, h // G, r] + ls
            z = scale * (kk @ q[s, h])
            a = np.exp(z - z.max())
            a /= a.sum()
            out[s, h], bulk[s, h] = a @ vv, a @ np.abs(vv)
            steep[s, h] = abs(scale) * (np.abs(kk) @ np.abs(q[s, h])).max()
    return out, bulk, steep, live


def tolerance(out, bulk, steep, live, D, dtype):
    """Half a step of the stored output, and to first order what fp32 arithmetic may add in front of it.  A logit is a sum of D products
    and a scaling, (D + 4) roundings of 2^-24 on the magnitudes; its error is one of the exponential's argument, whose own
    function adds 4 units, and acts on the weights above and below the fraction: twice.  Sums over the tokens, their rescalings and
    the joins of parts: no more than 2 roundings per token and 64 besides, above and below as well.  bf16 weights in two terms: 2^-9 * 2^-9."""
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    n = live[:, None, None]
    eps = 2.0 ** -24 * (2 * (D + 4) * np.maximum(steep, 1.0) + 2 * (2 * n + 64)) + (2.0 ** -18 if dtype == "bf16" else 0.0)
    return half * np.abs(out) + (1 + half) * eps * bulk + 1e-37


def write(k, v, sizes, new_k, new_v, new_sizes, seq, pos, table):
    """In place, k, v [n_pages, H, P, D]."""
    n_pages, _, P, _ = k.shape
    for t in range(len(pos)):
        s, p = (t if seq is None else int(seq[t])), int(pos[t])
        if not (0 <= s < table.shape[0] and 0 <= p < table.shape[1] * P):
            continue
        page = int(table[s, p // P])
        if not 0 <= page < n_pages:
            continue
        k[page, :, p % P], v[page, :, p % P] = new_k[t], new_v[t]
        if sizes is not None:
            sizes[page, p % P] = 1 if new_sizes is None else new_sizes[t]


def compact(pools, sizes, kept_idx, lengths, first, span, n_keep, table_in, table_out):
    """In place, pools [layers, n_pages, H, P, D].  Returns the lengths afterwards."""
    n_pages, P = pools[0].shape[1], pools[0].shape[3]
    before, before_s = [p.copy() for p in pools], None if sizes is None else sizes.copy()
    ends, at = [], 0
    for i in range(len(lengths)):
        f = first[i]
        survivors = list(range(f))
        survivors += [f + int(j) if 0 <= j < span[i] else None for j in kept_idx[at:at + n_keep[i]]]
        survivors += list(range(f + span[i], lengths[i]))
        at += n_keep[i]
        ends.append(len(survivors))
        for j, p in enumerate(survivors):
            if p is None:
                continue
            a, b = int(table_in[i][p // P]), int(table_out[i][j // P])
            if 0 <= a < n_pages and 0 <= b < n_pages:
                for pool, old in zip(pools, before):
                    pool[:, b, :, j % P] = old[:, a, :, p % P]
                if sizes is not None:
                    sizes[b, j % P] = before_s[a, p % P]
    return ends
