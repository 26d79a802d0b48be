"""What the serving-step calls are compared with: their definitions in include/awsrc.h
on the host, in whole numbers or 64 bits, without the library's code."""
import math
from fractions import Fraction

import torch


def plan(page, table, length, free, count, keep, add, n_tok):
    """Lists in, lists out: (table, length, free, count, q_start, tok_seq, tok_pos, tok_slot, flags)."""
    table, free, length = [list(r) for r in table], list(free), list(length)
    most, flags = len(table[0]) * page if table else 0, 0

    def pages(tokens):
        return -(-tokens // page)

    n = len(length)
    keep = list(length) if keep is None else list(keep)
    add = list(add)
    ok = [0 <= length[b] <= most and 0 <= keep[b] <= length[b] and add[b] >= 0 and keep[b] + add[b] <= most
          for b in range(n)]
    if not all(ok):
        flags |= 8
    for b in range(n):
        if not ok[b]:
            keep[b], add[b] = length[b], 0
    grow = [pages(keep[b] + add[b]) - pages(length[b]) if ok[b] else 0 for b in range(n)]
    room = count + sum(max(0, -g) for g in grow)
    need = tokens = 0
    for b in range(n):
        need, tokens = need + max(0, grow[b]), tokens + add[b]
        if (grow[b] > 0 and need > room) or tokens > n_tok:
            if add[b] > 0:
                flags |= 16
            add[b] = 0  # they still count for those behind
    back = [(b, j) for b in range(n) if ok[b] for j in range(pages(keep[b] + add[b]), pages(length[b]))]
    if not 0 <= count <= len(free) or count + len(back) > len(free):
        return table, length, free, count, [0] * (n + 1), [-1] * n_tok, [-1] * n_tok, [-1] * n_tok, flags | 8
    for b, j in back:
        free[count] = table[b][j]
        count += 1
    q_start, seq, pos, slot = [0], [], [], []
    for b in range(n):
        for j in range(pages(length[b]), pages(keep[b] + add[b])) if ok[b] else ():
            count -= 1
            table[b][j] = free[count]
        for p in range(keep[b], keep[b] + add[b]):
            seq.append(b)
            pos.append(p)
            slot.append(table[b][p // page] * page + p % page)
        length[b] = keep[b] + add[b]
        q_start.append(len(seq))
    behind = [-1] * (n_tok - len(seq))
    return table, length, free, count, q_start, seq + behind, pos + behind, slot + behind, flags


def units(p):
    """A probability in units of 2^-45, rounded to nearest even."""
    if math.isnan(p) or p <= 0:
        return 0
    return round(Fraction(min(p, 1.0)) * 2 ** 45)


def clean(p):
    return 0.0 if math.isnan(p) or p <= 0 else min(p, 1.0)


def verify(row_start, ids, target, draft, u, r, max_draft, kv_len):
    """Lists of lists in (rows of Python floats), (accepted, tokens, keep, flags) out."""
    n_rows, vocab, flags = len(ids), len(target[0]), 0
    accepted, tokens, keep = [], [], []
    for b in range(len(row_start) - 1):
        first, end = row_start[b], row_start[b + 1]
        if not 0 <= first <= end <= n_rows or end - first - 1 > max_draft or end == first:
            if not (first >= 0 and first == end <= n_rows):
                flags |= 8
            accepted.append(0)
            tokens.append([-1] * (max_draft + 1))
            keep.append(kv_len[b])
            continue
        t, got = first, []
        while t < end - 1:
            x = ids[t + 1]
            if not 0 <= x < vocab:
                break
            q = 1.0 if draft is None else clean(draft[t][x])
            ut = 0.0 if math.isnan(u[t]) else max(0.0, u[t])
            if math.isinf(ut) or not Fraction(ut) * Fraction(q) < Fraction(clean(target[t][x])):
                break
            got.append(x)
            t += 1
        # ids outside the vocabulary are reported wherever they stand among the first group that is looked at
        if any(not 0 <= x < vocab for x in ids[first + 1:end]):
            flags |= 8
        full = [units(p) for p in target[t]]
        w = full
        if t < end - 1:
            if draft is None:
                w = [0 if j == ids[t + 1] else f for j, f in enumerate(full)]
            else:
                w = [max(0, f - units(q)) for f, q in zip(full, draft[t])]
            if not any(w):
                w = full
        total = sum(w)
        rb = 0.0 if math.isnan(r[b]) else max(0.0, r[b])
        bar = Fraction(rb) * total if rb < 1 else total - Fraction(1, 2)  # the largest r below 1 reaches the last weight
        at, token = 0, -1
        for j, v in enumerate(w):
            at += v
            if v and at > bar:
                token = j
                break
        accepted.append(len(got))
        tokens.append((got + [token] + [-1] * max_draft)[:max_draft + 1])
        keep.append(kv_len[b] - (end - 1 - t))
    return accepted, tokens, keep, flags


def e4m3(x):
    """Nearest e4m3 value, ties to even; |x| <= 448."""
    _, p = torch.frexp(x)
    step = torch.ldexp(torch.ones((), dtype=torch.float64), (p - 4).clamp(min=-9))
    return torch.round(x / step) * step


def quantize(x):
    """float64 [rows, cols] on the CPU: (code values [rows, cols], exponents [rows, blocks]); a block that is not finite has
    NaN codes and exponent 0."""
    rows, cols = x.shape
    codes, exps = torch.empty_like(x), torch.zeros(rows, -(-cols // 128), dtype=torch.int32)
    for a in range(0, cols, 128):
        part = x[:, a:a + 128]
        for i in range(rows):
            row = part[i]
            if not bool(torch.isfinite(row).all()):
                codes[i, a:a + 128] = math.nan
                continue
            most, e = float(row.abs().max()), -64
            while most > 448 * 2.0 ** e:
                e += 1
            exps[i, a // 128] = e
            codes[i, a:a + 128] = e4m3(row * 2.0 ** -e)
    return codes, exps


def place(codes, exps):
    """The byte layouts from include/awsrc.h, written out: codes as float64 [B, R, 128], e + 127 as [.., .., 32, 4, 4]; places that no
    element has stay 0."""
    rows, cols = codes.shape
    blocks = exps.shape[1]
    c = torch.zeros(blocks, -(-rows // 8) * 8, 128, dtype=torch.float64)
    e = torch.zeros(-(-blocks // 4), -(-rows // 128), 32, 4, 4, dtype=torch.uint8)
    k = torch.arange(cols)
    for r in range(rows):
        c[k // 128, r, 16 * ((k % 128 // 16) ^ (r % 8)) + k % 16] = codes[r]
        for b in range(blocks):
            e[b // 4, r // 128, r % 32, r % 128 // 32, b % 4] = int(exps[r, b]) + 127
    return c, e
