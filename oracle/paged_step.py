"""The decoding step on a paged fp8 cache, written out in fp64 / plain integers (test
infrastructure; shares no code with the GPU path).  Everything goes request by request,
token by token: no prefix sums, no tiles, no bit tricks."""
from __future__ import annotations

import math

import numpy as np

from .oracle import e4m3_decode

# the 127 non-negative finite E4M3 values, ascending, and their codes
_VALUES = np.asarray([e4m3_decode(c) for c in range(127)])
DECODE = np.asarray([e4m3_decode(c) for c in range(256)])


def e4m3_encode(x):
    """Codes of fp64 values: nearest, ties to the even code, saturating; NaN to 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    a = np.where(np.isnan(a), 0.0, a)
    i = np.clip(np.searchsorted(_VALUES, a), 1, 126)
    down, up = a - _VALUES[i - 1], _VALUES[i] - a
    i = np.where((down < up) | ((down == up) & (i % 2 == 1)), i - 1, i)
    return np.where(np.isnan(x), 0x7F, i + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def plan_pages(page_size, pages_per_seq, n_pages, max_new, kv_len, n_new, held, n_free, free_pages, table):
    """(table, new_kv_len, new_held, new_n_free, token_start, slot_map, refused) of lvspec_plan_pages."""
    table = np.array(table)
    kv_len, n_new, held = [list(map(int, a)) for a in (kv_len, n_new, held)]
    n_free = min(max(int(n_free), 0), n_pages)
    top, wanted, at, refused = n_free, 0, 0, False
    new_len, new_held, starts, slots = [], [], [], [-1] * max_new
    for b, (length, new, have) in enumerate(zip(kv_len, n_new, held)):
        starts.append(min(at, 2**31 - 1))
        first, at = at, at + max(new, 0)
        good = length >= 0 and new >= 0 and 0 <= have <= pages_per_seq and length + new <= pages_per_seq * page_size \
            and at <= max_new
        need = max(0, math.ceil((length + new) / page_size) - have) if good else 0
        wanted += need
        if need and wanted > n_free:
            good = False
        if good:
            for j in range(need):
                top -= 1
                table[b, have + j] = free_pages[top]
            for i in range(new):
                page = int(table[b, (length + i) // page_size])
                if 0 <= page < n_pages:
                    slots[first + i] = page * page_size + (length + i) % page_size
        refused |= not good
        new_len.append(length + new if good else length)
        new_held.append(have + need if good else have)
    starts.append(min(at, 2**31 - 1))
    return table, new_len, new_held, top, starts, slots, refused


def append(x, slots, pool, scale, page_size, block):
    """(pool, scale) after the rows x [n, Hkv, D] (fp64) went to their slots: codes uint8
    [n_pages, Hkv, page_size, D], scales fp32 [n_pages, Hkv, page_size / block]."""
    pool, scale = np.array(pool), np.array(scale)
    n_pages, heads = pool.shape[:2]
    groups = {}
    for i, s in enumerate(np.asarray(slots).tolist()):
        if 0 <= s < n_pages * page_size:
            groups.setdefault(s // block, []).append(i)
    for tokens in groups.values():
        s0 = int(slots[tokens[0]])
        page, part = s0 // page_size, s0 % page_size // block
        begun = min(int(slots[i]) % block for i in tokens)
        for h in range(heads):
            finite = np.abs(x[tokens, h])
            a = np.max(finite, where=np.isfinite(finite), initial=0.0)
            # the smallest power of two that brings a to at most 448, counted up or down
            k = -100
            if a > 0:
                k = math.floor(math.log2(a / 448.0)) - 2
                while a > 448.0 * 2.0 ** k:
                    k += 1
                k = min(max(k, -100), 119)
            s = np.float32(2.0 ** k)
            old = scale[page, h, part]
            first = part * block
            if begun > 0:
                s = max(s, old)
                if s != old:
                    part_codes = pool[page, h, first:first + begun]
                    ratio = np.float64(np.float32(old) / np.float32(s))
                    pool[page, h, first:first + begun] = e4m3_encode(np.float32(DECODE[part_codes] * ratio))
            scale[page, h, part] = s
            for i in tokens:
                with np.errstate(invalid="ignore"):
                    pool[page, h, int(slots[i]) % page_size] = e4m3_encode(np.float32(np.float32(x[i, h]) / s))
    return pool, scale


def attention(q, k_pool, v_pool, k_scale, v_scale, table, kv_len, span, block, branch_len=0, absolute=False):
    """(out, mass) in fp64.  q fp64 [B, gamma, Hq, D]; pools uint8 [n_pages, Hkv, page_size, D].
    absolute: the probabilities' product with |v| instead."""
    B, gamma, Hq, D = q.shape
    n_pages, Hkv, page_size, _ = k_pool.shape
    bl = branch_len or gamma
    out, mass = np.zeros((B, gamma, Hq, D)), np.zeros((B, gamma, Hq))
    for b in range(B):
        L = int(kv_len[b])
        if L <= 0:
            continue
        at = np.arange(L)
        pages, off = np.asarray(table[b])[at // page_size], at % page_size
        there = (pages >= 0) & (pages < n_pages)
        pg = np.where(there, pages, 0)
        tail = at - (L - gamma)
        inside = (at >= span[b][0]) & (at < span[b][1])
        for h in range(Hkv):
            k = DECODE[k_pool[pg, h, off]] * k_scale[pg, h, off // block][:, None].astype(np.float64)
            v = DECODE[v_pool[pg, h, off]] * v_scale[pg, h, off // block][:, None].astype(np.float64)
            k[~there] = 0
            v[~there] = 0
            for g in range(gamma):
                sees = (tail <= g) & ((tail < 0) | (tail // bl == g // bl))
                if not sees.any():
                    continue
                for hq in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                    s = (k[sees] @ q[b, g, hq]) / math.sqrt(D)
                    e = np.exp(s - s.max())
                    p = e / e.sum()
                    out[b, g, hq] = p @ (np.abs(v[sees]) if absolute else v[sees])
                    mass[b, g, hq] = p[inside[sees]].sum()
    return out, mass


def kept_tokens(logits, T, top_k, top_p, min_p):
    """(tokens in falling order that the filters keep, all weights in fp64) of one row; T > 0."""
    l = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    order = sorted(range(len(l)), key=lambda i: (-l[i], i))
    top = l[order[0]]
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(l == top, 1.0, np.exp((l - top) / T))
    w = np.where(l == -np.inf, 0.0, w) if top > -np.inf else w
    kept = order[:top_k] if 0 < top_k < len(l) else order
    if top_p < 1:
        share, total, n = 0.0, math.fsum(w[i] for i in kept), 0
        for i in kept:
            if n and share >= max(top_p, 0.0) * total:
                break
            share += w[i]
            n += 1
        kept = kept[:n]
    if min_p > 0:
        limit = top + T * math.log(min(min_p, 1.0))
        kept = [i for i in kept if l[i] >= limit]
    return kept, w


def sample(logits, T, top_k, top_p, min_p, u):
    """(token, probability, how far u is from the nearest border of the token's interval)."""
    l = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    if not T > 0 or not l.max() > -np.inf:
        return (int(l.argmax()) if l.max() > -np.inf else 0), 1.0, 1.0
    kept, w = kept_tokens(logits, T, top_k, top_p, min_p)
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    total = math.fsum(w[i] for i in kept)
    run = 0.0
    for i in sorted(kept):
        if w[i] > 0 and run + w[i] > u * total:
            return i, w[i] / total, min(u - run / total if run else 1.0, (run + w[i]) / total - u if run + w[i] < total else 1.0)
        run += w[i]
    raise AssertionError
