"""CPU oracle of the 8-bit KV cache and of the page tables of rows that grow: plain numpy in 64 bits.

TEST INFRASTRUCTURE ONLY, as dag_oracle: it shares no code with the HIP path and never imports it.

  * Codes are e4m3 (sign, 4 bits of exponent with bias 7, 3 of mantissa; no infinity, largest value 448); a code c of a page stands
    for scale * c.  Arrays here are indexed by token: codes [page][head][slot][dim], scales [page][head].
  * The scale of a page and head is the smallest power of two, 2^-100 at least, with which all its tokens so far are within
    +-448; when it grows the codes that are there are divided by the same factor and rounded again.
"""
import math

import numpy as np

from oracle import dag_oracle as orc

PAGE = 16
TOP = 448.0


def e4m3(x):
    """To the nearest value of the format, ties to even (|x| up to 448)."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(x / step) * step


def scale_for(most):
    k = -100
    while most > TOP * 2.0 ** k:
        k += 1
    return 2.0 ** k


def tokens_of_pools(k_pool, v_pool):
    """Pools as the library stores them (float arrays) -> codes [page][head][slot][dim]."""
    p, h, _, _, _ = k_pool.shape
    k = np.asarray(k_pool, dtype=np.float64).transpose(0, 1, 3, 2, 4).reshape(p, h, PAGE, -1)
    return k, np.asarray(v_pool, dtype=np.float64).transpose(0, 1, 3, 2).copy()


def append(codes, scales, x, slots):
    """Stores x [token][head][dim] at `slots`, in place.  Returns the exact value that every element of a touched page was
    rounded from: [(page, first slot of the run, values [head][slot][dim])]."""
    n_pages, heads = scales.shape
    runs = []
    for t, s in enumerate(slots):
        s = int(s)
        if s < 0 or s >= n_pages * PAGE:
            continue
        if runs and s % PAGE and runs[-1][1][-1] == (t - 1, s - 1):
            runs[-1][1].append((t, s))
        else:
            runs.append((s // PAGE, [(t, s)]))
    touched = []
    for page, run in runs:
        i0 = run[0][1] % PAGE
        exact = np.zeros((heads,) + codes.shape[2:])
        for h in range(heads):
            new = np.stack([x[t, h] for t, _ in run])
            fine = new[np.isfinite(new)]
            scale = scale_for(np.abs(fine).max() if fine.size else 0.0)
            if i0 == 0:
                codes[page, h] = 0.0
            else:
                scale = max(scale, scales[page, h])
                exact[h] = codes[page, h] * scales[page, h]
                codes[page, h] = e4m3(codes[page, h] * (scales[page, h] / scale))
            for t, s in run:
                exact[h, s % PAGE] = x[t, h]
                codes[page, h, s % PAGE] = np.where(np.isfinite(x[t, h]), e4m3(np.where(np.isfinite(x[t, h]), x[t, h], 0) / scale), np.nan)
            scales[page, h] = scale
        touched.append((page, i0, exact))
    return touched


def attention(q, contexts, k, v, scale):
    """softmax(scale q . K^T) V for every row over its context, a list of (pages, tokens of them that it sees).  k, v: values
    [page][head][slot][dim].  Returns the result, the same with |V| in the place of V, and the largest sum_d |q_d k_d| * |scale| of a row."""
    rows, hq, d = q.shape
    hkv = k.shape[1]
    out, mass, size = np.zeros((rows, hq, d)), np.zeros((rows, hq, d)), np.zeros((rows, hq, 1))
    for r in range(rows):
        for h in range(hkv):
            parts = [(k[pages, h].reshape(-1, d)[:n], v[pages, h].reshape(-1, d)[:n]) for pages, n in contexts[r] if n > 0]
            if not parts:
                continue
            keys, vals = np.concatenate([a for a, _ in parts]), np.concatenate([b for _, b in parts])
            for j in range(h * hq // hkv, (h + 1) * hq // hkv):
                s = keys @ q[r, j] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[r, j], mass[r, j], size[r, j] = p @ vals, p @ np.abs(vals), (np.abs(keys) @ np.abs(q[r, j])).max() * abs(scale)
    return out, mass, size


def release(table, free, count, row_len, ended):
    """In place; returns the new number of free pages."""
    for r in range(len(row_len)):
        if ended[r]:
            for p in table[r, :min(-(-max(int(row_len[r]), 0) // PAGE), table.shape[1])]:
                free[count] = p
                count += 1
            row_len[r] = 0
    return count


def extend(table, free, count, row_len, new_len, pos0):
    """In place, row by row and token by token.  Returns (free pages left, new_off, slots, pos, page_off, pages, refused)."""
    width = table.shape[1]
    asked = taken = refused = 0
    new_off, slots, pos, page_off, pages = [0], [], [], [0], []
    for r in range(len(row_len)):
        n, w = max(int(row_len[r]), 0), max(int(new_len[r]), 0)
        need = math.ceil((n + w) / PAGE) - math.ceil(n / PAGE)
        fits = n + w <= width * PAGE
        ok = fits and (need == 0 or asked + need <= count)
        for j in range(w):
            at = n + j
            if ok and at % PAGE == 0:
                table[r, at // PAGE] = free[count - 1 - (asked + at // PAGE - math.ceil(n / PAGE))]
            slots.append(table[r, at // PAGE] * PAGE + at % PAGE if ok else -1)
            pos.append(pos0[r] + at)
        asked += need if fits else 0
        taken += need if ok else 0
        refused += not ok and w > 0
        row_len[r] = n + (w if ok else 0)
        new_off.append(new_off[-1] + w)
        pages += list(table[r, :math.ceil(row_len[r] / PAGE)])
        page_off.append(len(pages))
    return count - taken, new_off, slots, pos, page_off, pages, refused


def rope(x, pos, theta):
    return orc.rope(x, pos, theta)


def fork(table, free, count, row_len, extra, parent, child, fork_len):
    """In place, fork by fork.  Returns (free pages left, copy_src, copy_dst, refused)."""
    before = np.maximum(np.asarray(row_len), 0).copy()
    taken, asked, refused, src, dst = set(), 0, 0, [], []
    for f, (p, c) in enumerate(zip(parent, child)):
        src.append(-1)
        dst.append(-1)
        if not (0 <= p < len(before) and 0 <= c < len(before)) or before[c] > 0 or c in taken:
            refused += 1
            continue
        taken.add(c)
        n = min(before[p], table.shape[1] * PAGE)
        n = n if fork_len is None else min(n, max(fork_len[f], 0))
        if n % PAGE:
            asked += 1
            if asked > count:
                refused += 1
                continue
            src[f], dst[f] = table[p, n // PAGE], free[count - asked]
        for i in range(n // PAGE):
            table[c, i] = table[p, i]
            if 0 <= table[p, i] < len(extra):
                extra[table[p, i]] += 1
        if n % PAGE:
            table[c, n // PAGE] = dst[f]
        row_len[c] = n
    return count - min(asked, count), src, dst, refused


def release_shared(table, free, count, row_len, extra, ended):
    """In place; returns the new number of free pages."""
    given = [int(p) for r in range(len(row_len)) if ended[r] for p in table[r, :min(-(-max(int(row_len[r]), 0) // PAGE), table.shape[1])]]
    given = [p for p in given if 0 <= p < len(extra)]
    for i, p in enumerate(given):
        if p not in given[i + 1:] and given.count(p) > max(extra[p], 0):
            free[count] = p
            count += 1
    for p in set(given):
        extra[p] = max(max(extra[p], 0) - given.count(p), 0)
    for r in range(len(row_len)):
        if ended[r]:
            row_len[r] = 0
    return count


def compact(table, free, count, row_len, extra):
    """Returns (table, free, extra, page_map, pairs)."""
    n = len(extra)
    none = set(int(p) for p in free[:count])
    used = n - count
    to = [p for p in range(used) if p in none]
    moved = [p for p in range(used, n) if p not in none]
    new = {p: p for p in range(used) if p not in none}
    new.update(zip(moved, to))
    table, free, holders = table.copy(), free.copy(), np.zeros(n, dtype=np.int64)
    for r in range(len(row_len)):
        for i in range(min(-(-max(int(row_len[r]), 0) // PAGE), table.shape[1])):
            table[r, i] = new.get(int(table[r, i]), table[r, i])
    for i in range(count):
        free[i] = n - 1 - i
    for p, q in new.items():
        holders[q] = extra[p]
    return table, free, holders, [new.get(p, -1) for p in range(n)], list(zip(moved, to))


def frequencies(rotary, theta, stretch=1.0, original=0.0, low=1.0, high=32.0):
    out = []
    for m in range(rotary // 2):
        f = theta ** (-2.0 * m / rotary)
        keep = 0.0 if original == 0 else min(max((original * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
        out.append(keep * f + (1 - keep) * f / stretch)
    return np.asarray(out)


def rotary(x, pos, freq, pairs, factor=1.0, transposed=False):
    """x [token][head][dim] in 64 bits: pair m turned by pos * freq[m], times factor."""
    y = np.array(x, dtype=np.float64)
    half = len(freq)
    i = 2 * np.arange(half) if pairs else np.arange(half)
    j = i + 1 if pairs else i + half
    angle = np.asarray(pos, dtype=np.float64)[:, None, None] * freq * (-1 if transposed else 1)
    c, s = np.cos(angle) * factor, np.sin(angle) * factor
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y
