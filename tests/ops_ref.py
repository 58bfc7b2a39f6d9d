"""Plain 64-bit forms of the paged cache and the block-scaled product (numpy, written from the
definitions in sbd.h; no code shared with the library), and the error bounds that follow from the
types the kernels compute in."""
import math

import numpy as np
import torch

from oracle import sbd_oracle as O

VALUES = O.decode_e4m3(np.arange(256)).astype(np.float64)   # value of each code, NaN for 0x7f and 0xff
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def f64(t):
    return t.detach().double().cpu().numpy()


def exponent(x):
    """Smallest e in [-100, 100] with |x| <= 448 * 2^e for every finite x, by trying every e."""
    x = np.abs(x[np.isfinite(x)])
    top = float(x.max()) if x.size else 0.0
    for e in range(-100, 101):
        if top <= math.ldexp(448.0, e):
            return e
    return 100


def round8(y):
    """Nearest e4m3 value (ties to the even code), saturating; NaN stays NaN."""
    return O.round_to_e4m3(np.asarray(y, np.float64), 0)


def plan(table, held, cached, free_list, free_count, n_new, release, rows, page):
    """sbd_paged_plan on host arrays; returns the updated state and (row_start, kv_len, slots)."""
    table, held, cached, free = (np.array(x, np.int64) for x in (table, held, cached, free_list))
    B, W = table.shape
    stack = [int(p) for p in free[:free_count]]
    free = free.copy()
    for b in range(B):
        if release is not None and release[b]:
            stack += [int(p) for p in table[b, :held[b]]]
            table[b], held[b], cached[b] = -1, 0, 0
    free[free_count:len(stack)] = stack[free_count:]
    kv, got, asked = np.zeros(B, np.int64), [], 0
    for b in range(B):
        total = int(cached[b]) + int(n_new[b])
        if cached[b] < 0 or n_new[b] < 0 or total > W * page:
            continue
        need = max(0, -(-total // page) - int(held[b]))
        if need and asked + need > len(stack):
            asked += need
            continue
        asked += need
        got.append((b, need))
        kv[b] = total
    taken = sum(n for _, n in got)
    pages = stack[len(stack) - taken:]
    at = 0
    for b, need in got:
        table[b, held[b]:held[b] + need] = pages[at:at + need]
        held[b] += need
        at += need
    starts = np.concatenate([[0], np.cumsum(np.maximum(n_new, 0))]).astype(np.int64)
    slots = np.full(rows, -1, np.int64)
    for b in range(B):
        for j in range(max(0, int(n_new[b]))):
            if starts[b] + j < rows and kv[b]:
                p = int(cached[b]) + j
                slots[starts[b] + j] = table[b, p // page] * page + p % page
    return table, held, cached, free, len(stack) - taken, starts, kv, slots


def append(codes, exps, x, starts, slots, page):
    """sbd_paged_append of one of keys and values: codes [pages][heads][page][dim] as values,
    updated in place with exps."""
    for b in range(len(starts) - 1):
        r, end = int(starts[b]), min(int(starts[b + 1]), len(slots))
        while r < end and slots[r] >= 0:
            pg, off = divmod(int(slots[r]), page)
            m = min(page - off, end - r)
            for h in range(x.shape[1]):
                e = exponent(x[r:r + m, h])
                if off:
                    e = max(e, int(exps[pg, h]))
                    codes[pg, h, :off] = round8(codes[pg, h, :off] * 2.0 ** (int(exps[pg, h]) - e))
                exps[pg, h] = e
                codes[pg, h, off:off + m] = round8(x[r:r + m, h] / 2.0 ** e)
            r += m


def attend(q, k_codes, v_codes, k_exp, v_exp, table, starts, kv_len, n_causal, scale, page, out_type, only=None):
    """(out, bound): float64 attention of every row (of `only`, if given), and how far the kernel
    may be from it.

    Bound, from the kernel's arithmetic: the weights are fp16 and held as 2^11 times a power of
    two that is at most the row's largest, so they are off by 2^-11 of themselves or by half of
    fp16's smallest step, 2^-25 / 2^11 = 2^-36 of the row's largest; a score is a
    sum of dim exact products in fp32 (off by dim * 2^-24 of the sum of their sizes, and by two
    roundings of 2^-24 where it is scaled and the maximum is taken off), an exponential is off
    by 2^-22 of itself; the sums of weights and outputs are fp32 (each of N terms adds 2^-24 of
    the whole); the result is rounded once to its type."""
    rows, nq, dh = q.shape
    H = k_exp.shape[1]
    k_all = VALUES[k_codes] * 2.0 ** k_exp.astype(np.float64)[:, :, None, None]
    v_all = (VALUES[v_codes] * 2.0 ** v_exp.astype(np.float64)[:, :, None, None]).transpose(0, 1, 3, 2)
    out, bound = np.zeros((rows, nq, dh)), np.zeros((rows, nq, dh))
    for b in range(len(starts) - 1):
        n, L = int(starts[b + 1] - starts[b]), int(kv_len[b])
        if n == 0 or L < n:
            continue
        pos = np.arange(L)
        pages = table[b, pos // page]
        known = (pages >= 0) & (pages < k_exp.shape[0])
        pages = np.where(known, pages, 0)
        for j in range(n):
            if starts[b] + j >= rows or (only is not None and starts[b] + j not in only):
                continue
            end = L - n + j + 1 if (n_causal is None or j < n_causal[b]) else L
            see = known & (pos < end)
            if not see.any():
                continue
            for h in range(nq):
                g = h // (nq // H)
                kk, vv = k_all[pages[see], g, pos[see] % page], v_all[pages[see], g, pos[see] % page]
                x = q[starts[b] + j, h]
                s = kk @ x * scale
                size = np.abs(kk) @ np.abs(x) * abs(scale)
                p = np.exp(s - s.max())
                w = p / p.sum()
                N = see.sum()
                o = w @ vv
                out[starts[b] + j, h] = o
                ds = size.max() * (dh + 3) * 2.0 ** -24 + np.abs(s).max() * 2.0 ** -23
                rel = 2.0 ** -11 + 2 * ds + 2.0 ** -21 + (N + 70) * 2.0 ** -23
                bound[starts[b] + j, h] = (rel * (w @ np.abs(vv)) + 2.0 ** -36 * np.abs(vv).sum(0)
                                           + HALF_STEP[out_type] * np.abs(o) * 1.01)
    return out, bound


def matmul(a, a_scale, b, b_scale, out_type, cols=None):
    """(out, bound) of the block-scaled product: fp32 sums of exact products, 128 and then one for
    each block, two roundings for the scales, one rounding of the result.  The matrix instruction
    of the 16-bit outputs cuts each of eight neighbouring products off at 2^-13 of the power of
    two of the largest (at most the largest itself): 8 * 2^-13 of the largest for each group.
    cols: which columns of the whole product the rows of b are (their scales' blocks)."""
    A, B = VALUES[a], VALUES[b]
    (m, k), n = A.shape, B.shape[0]
    kb = -(-k // 128)
    out, size, cut = np.zeros((m, n)), np.zeros((m, n)), np.zeros((m, n))
    for c in range(kb):
        s = slice(128 * c, min(k, 128 * c + 128))
        f = a_scale[c].astype(np.float64)[:, None] * b_scale[:, c].astype(np.float64)[(np.arange(n) if cols is None else cols) // 128]
        out += (A[:, s] @ B[:, s].T) * f
        size += (np.abs(A[:, s]) @ np.abs(B[:, s]).T) * np.abs(f)
        if out_type != torch.float32:
            for i in range(s.start, s.stop, 8):
                top = np.zeros((m, n))
                for j in range(i, min(i + 8, s.stop)):
                    np.maximum(top, np.abs(A[:, j])[:, None] * np.abs(B[:, j])[None, :], out=top)
                cut += top * 2.0 ** -10 * np.abs(f)
    bound = cut + size * (128 + kb + 4) * 2.0 ** -24 + HALF_STEP[out_type] * np.abs(out) * 1.01
    top = float(torch.finfo(out_type).max)  # what exceeds the type is infinite in it
    return np.where(np.abs(out) > top, np.copysign(np.inf, out), out), bound


def worst(got, want, bound):
    """Largest error as a share of its bound (NaN in the same places, or infinite)."""
    if not np.array_equal(np.isnan(got), np.isnan(want)):
        return math.inf
    with np.errstate(invalid="ignore"):
        d = np.abs(got - want)
    d = np.where(np.isnan(want) | (got == want), 0.0, d)
    return float(np.max(np.where(d == 0, 0.0, d / np.maximum(np.nan_to_num(bound, nan=1.0), 1e-300)), initial=0.0))
