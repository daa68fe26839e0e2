"""Plain model of the paged 8-bit cache, in Python and numpy, 64 bits: written from the definitions in include/pq_attn.h, token by
token and block by block.  Test infrastructure only; shares nothing with the kernels."""
from __future__ import annotations

from fractions import Fraction

import numpy as np

FLOOR = 127.0 * 2.0 ** -40


# ------------------------------------------------------------------------------------------------------------- plan

def plan(n_new, seq_len, free_list, free_count, table, block, n_tokens):
    """The step of pq_paged_plan, request after request.  free_list and table are copied.  Returns a dict of its outputs."""
    free, table = list(map(int, free_list)), np.array(table)
    n_blocks, most = len(free), table.shape[1] * block
    count = min(max(int(free_count), 0), n_blocks)
    old = [min(max(int(n), 0), most) for n in seq_len]
    length, got, start, slots = [], [], [0], np.full(n_tokens, -1, np.int64)
    for b, n in enumerate(n_new):
        if n < 0:
            for j in range(-(-old[b] // block)):
                if count < n_blocks:
                    free[count] = int(table[b, j])
                    count += 1
    asked_blocks, top, refused = 0, count, False
    for b, n in enumerate(n_new):
        n = max(int(n), 0)
        first = start[-1]
        start.append(first + n)
        give = 0
        if n > 0 and old[b] + n <= most and first + n <= n_tokens:
            used = -(-old[b] // block)
            need = -(-(old[b] + n) // block) - used
            asked_blocks += need
            if need == 0 or asked_blocks <= count:
                give = n
                for j in range(need):
                    top -= 1
                    table[b, used + j] = free[top]
                for i in range(n):
                    p = old[b] + i
                    held = int(table[b, p // block])
                    if 0 <= held < n_blocks:
                        slots[first + i] = held * block + p % block
        refused |= give != n
        got.append(give)
        length.append(0 if n_new[b] < 0 else old[b] + give)
    return {"new_seq_len": np.array(length), "new_free_count": np.array([top]), "tok_start": np.minimum(start, n_tokens),
            "tok_len": np.array(got), "slot_map": slots, "block_table": table, "free_list": np.array(free),
            "refused": refused}


# ------------------------------------------------------------------------------------------------ blocks held together

def _lengths(seq_len, table, block):
    return [min(max(int(n), 0), table.shape[1] * block) for n in seq_len]


def fork(parent, keep, seq_len, free_list, free_count, table, holders, block):
    """pq_paged_fork, request after request.  Nothing given is changed.  Returns a dict of its outputs, and what it reports."""
    table, holders, free = np.array(table), np.array(holders), list(map(int, free_list))
    n_blocks, old, before = len(free), _lengths(seq_len, table, block), np.array(table)
    count = min(max(int(free_count), 0), n_blocks)
    top, asked = count, 0
    length, src, dst, refused, outside = list(old), [], [], False, False
    for b, p in enumerate(map(int, parent)):
        pair = (-1, -1)
        if p >= 0 and p != b:
            if p >= len(old) or old[b] != 0:
                refused = True
            else:
                n = old[p] if keep is None else max(0, min(old[p], int(keep[b])))
                full, last = n // block, int(before[p, n // block]) if n % block else -1
                needs = n % block != 0 and 0 <= last < n_blocks
                asked += needs
                if needs and asked > count:
                    refused = True
                else:
                    for j in range(full):
                        x = table[b, j] = before[p, j]
                        if 0 <= x < n_blocks:
                            holders[x] += 1
                        else:
                            outside = True
                    if needs:
                        top -= 1
                        pair = (last, free[top])
                        table[b, full] = free[top]
                    elif n % block:
                        table[b, full], outside = last, True
                    length[b] = n
        src.append(pair[0])
        dst.append(pair[1])
    return {"new_seq_len": np.array(length), "new_free_count": np.array([top]), "block_table": table, "holders": holders,
            "copy_src": np.array(src), "copy_dst": np.array(dst), "refused": refused, "outside": outside}


def free(n_new, seq_len, free_list, free_count, table, holders, block):
    """pq_paged_free.  Nothing given is changed."""
    table, left, listed = np.array(table), np.array(holders, np.int64), np.array(free_list)
    n_blocks, old = len(listed), _lengths(seq_len, np.array(table), block)
    gone, over, outside = set(), False, False
    for b, n in enumerate(n_new):
        for x in map(int, table[b, :-(-old[b] // block)] if n < 0 else []):
            if not 0 <= x < n_blocks:
                outside = True
            elif x in gone:
                over = True
            elif left[x] > 0:
                left[x] -= 1
            else:
                gone.add(x)
    count = min(max(int(free_count), 0), n_blocks)
    for x in sorted(gone, reverse=True):
        if count < n_blocks:
            listed[count] = x
            count += 1
    return {"new_seq_len": np.array([0 if n < 0 else m for n, m in zip(n_new, old)]), "new_free_count": np.array([count]),
            "free_list": listed, "holders": left, "over": over, "outside": outside}


def compact(seq_len, free_list, free_count, table, holders, block):
    """pq_paged_compact.  Lists hold only what the call writes of them."""
    table, holders = np.array(table), np.array(holders)
    n_blocks, old = len(holders), _lengths(seq_len, table, block)
    listed = [int(x) for x in free_list[:min(max(int(free_count), 0), n_blocks)]]
    gone = {x for x in listed if 0 <= x < n_blocks}
    outside = len(gone) < len(set(listed))
    n_live = n_blocks - len(gone)
    src = [x for x in range(n_blocks - 1, n_live - 1, -1) if x not in gone]
    dst = [x for x in range(n_live) if x in gone]
    assert len(src) == len(dst)
    moved = {x: -1 if x in gone else x for x in range(n_blocks)} | dict(zip(src, dst))
    new_holders = np.zeros_like(holders)
    for x, to in moved.items():
        if to >= 0:
            new_holders[to] = holders[x]
    for b, n in enumerate(old):
        for j in range(-(-n // block)):
            x = int(table[b, j])
            if 0 <= x < n_blocks:
                table[b, j] = moved[x]
                outside |= moved[x] < 0
            else:
                outside = True
    return {"new_free_list": np.arange(n_blocks - 1, n_live - 1, -1), "new_free_count": np.array([len(gone)]),
            "new_block_table": table, "new_holders": new_holders, "moved_to": np.array([moved[x] for x in range(n_blocks)]),
            "copy_src": np.array(src, int), "copy_dst": np.array(dst, int), "n_copies": np.array([len(src)]), "outside": outside}


# ------------------------------------------------------------------------------------------------------------ cache

def nearest(x, s):
    """x / s to the nearest integer, ties to even, exactly."""
    return round(Fraction(float(x)) / Fraction(float(s)))


def nearest_all(x, s):
    """`nearest` of an array: where the quotient in double is away from a tie it decides, else the exact one does."""
    x = np.asarray(x, np.float64)
    quotient = x / float(s)
    codes = np.rint(quotient)
    close = np.abs(np.abs(quotient - np.floor(quotient)) - 0.5) < 1e-9
    for at in zip(*np.nonzero(close)):
        codes[at] = nearest(x[at], s)
    return codes


class Cache:
    """Codes [n_blocks, Hkv, block, d] and scales [n_blocks, Hkv] of K or V."""

    def __init__(self, n_blocks, heads, block, dim):
        self.codes = np.zeros((n_blocks, heads, block, dim), np.int64)
        self.scale = np.zeros((n_blocks, heads), np.float32)

    def append(self, x, slots):
        """x [tokens, Hkv, d] in its storage type, slots [tokens]."""
        n_blocks, heads, block, dim = self.codes.shape
        x = np.asarray(x, np.float64)
        t = 0
        while t < len(slots):
            slot, n = int(slots[t]), 1
            if not 0 <= slot < n_blocks * block:
                t += 1
                continue
            while t + n < len(slots) and slots[t + n] == slot + n and (slot + n) % block:
                n += 1
            held, first = slot // block, slot % block
            for h in range(heads):
                new = x[t:t + n, h]
                was = self.scale[held, h] if first else np.float32(0)
                if not np.isfinite(new).all() or not np.isfinite(was):
                    self.scale[held, h] = np.nan
                    self.codes[held, h, first:first + n] = 0
                    continue
                s = max(np.float32(max(np.abs(new).max(), FLOOR) / 127.0), was)
                if first and s > was:
                    older = self.codes[held, h, :first] * float(was)            # exact
                    self.codes[held, h, :first] = nearest_all(older, s)
                self.codes[held, h, first:first + n] = np.clip(nearest_all(new, s), -127, 127)
                self.scale[held, h] = s
            t += n

    def bytes(self, values_layout):
        """What the device holds, uint8 [n_blocks, Hkv, block * d]."""
        c = (self.codes + 128).astype(np.uint8)
        n_blocks, heads, block, dim = c.shape
        if values_layout:
            c = c.reshape(n_blocks, heads, block // 16, 4, 4, dim // 64, 4, 16).transpose(0, 1, 2, 5, 3, 7, 6, 4)
        return np.ascontiguousarray(c).reshape(n_blocks, heads, block * dim)

    @staticmethod
    def from_bytes(data, scale, block, dim, values_layout):
        data = np.asarray(data)
        n_blocks, heads = data.shape[:2]
        cache = Cache(n_blocks, heads, block, dim)
        if values_layout:
            data = data.reshape(n_blocks, heads, block // 16, dim // 64, 4, 16, 4, 4).transpose(0, 1, 2, 4, 7, 3, 6, 5)
        cache.codes = data.reshape(n_blocks, heads, block, dim).astype(np.int64) - 128
        cache.scale = np.array(scale, np.float32)
        return cache

    def rows(self, table_row, n):
        """Values of a sequence's first n tokens, [Hkv, n, d], and which of them the cache holds."""
        n_blocks, heads, block, dim = self.codes.shape
        out, there = np.zeros((heads, n, dim)), np.zeros(n, bool)
        for j in range(-(-n // block)):
            held, upto = int(table_row[j]), min(n, (j + 1) * block)
            if 0 <= held < n_blocks:
                part = self.codes[held, :, :upto - j * block] * self.scale[held].astype(np.float64)[:, None, None]
                out[:, j * block:upto], there[j * block:upto] = part, True
        return out, there


# -------------------------------------------------------------------------------------------------------- attention

def attention(q, k, v, there, scale, sees):
    """q [rows, Hq, d], k and v [Hkv, n, d]; row r attends over those of the first sees[r] tokens that are there.

    Returns out [rows, Hq, d], sum_t p_t |v_t| of the same shape, and for each row and head the largest sum_i |q_i k_i| *
    scale and the number of tokens times the largest p_t max_d |v_t| — what the bounds of an implementation in fewer bits
    are made of."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    rows, heads, dim = q.shape
    group = heads // k.shape[0]
    out, spread, size, peak = np.zeros(q.shape), np.zeros(q.shape), np.zeros((rows, heads)), np.zeros((rows, heads))
    for r in range(rows):
        n = max(0, min(int(sees[r]), k.shape[1]))
        use = there[:n]
        if not use.any():
            continue
        for h in range(heads):
            kk, vv = k[h // group, :n][use], v[h // group, :n][use]
            t = kk @ q[r, h] * scale
            p = np.exp(t - t.max())
            p /= p.sum()
            out[r, h], spread[r, h] = p @ vv, p @ np.abs(vv)
            size[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)
            peak[r, h] = (p * np.abs(vv).max(-1)).max() * len(p)
    return out, spread, size, peak
