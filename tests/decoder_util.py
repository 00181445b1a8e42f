"""Inputs for the tests of the decoder attention, made with numpy from a seed."""
import math

import numpy as np

import oracle
from paper_2101_01321_amd import binding as B


def dyadic(real):
    return B.ibert_dyadic_from_double(real).tuple()


def normal8(rng, std, *shape):
    return np.clip(np.rint(rng.normal(0, std, shape)), -127, 127).astype(np.int8)


def scattered_table(rng, lens, page, width=None, spare=3):
    """A block table whose pages lie anywhere in the cache; entries that no sequence needs name pages too (they are never read)."""
    need = [-(-int(n) // page) for n in lens]
    width = max(1, max(need, default=0)) if width is None else width
    total = sum(need) + spare
    pool = rng.permutation(total)
    table = rng.integers(0, total, (len(lens), width)).astype(np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pool[at:at + n]
        at += n
    return table, total


class Attention:
    """One call of ibert_paged_attention_i: n[b] query rows on kv[b] keys.  pad: rows of no sequence behind the last; ld: columns
    behind those of a row."""

    def __init__(self, seed, hq, hk, D, page, n, kv, window=0, sinks=0, std=32.0, scale=6.0 / 127, pad=0, ld=0, out_scale=1 / 3):
        rng = np.random.default_rng(seed)
        self.hq, self.hk, self.D, self.page, self.window, self.sinks = hq, hk, D, page, window, sinks
        self.n, self.kv = np.array(n, np.int64), np.array(kv, np.int64)
        self.batch, self.rows = len(n), int(self.n.sum()) + pad
        self.table, self.pages = scattered_table(rng, self.kv, page)
        cells = self.pages * page * hk * D
        self.q, self.k, self.v = normal8(rng, std, self.rows, hq * D + ld), normal8(rng, std, cells), normal8(rng, std, cells)
        self.q_start = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.kv_len = self.kv.astype(np.int32)
        self.s_dy = dyadic(scale * scale / math.sqrt(D) * 64 / math.log(2))
        self.o_dy = dyadic(1 / out_scale / 65536)
        self.out = rng.integers(-127, 128, (self.rows, hq * D + ld)).astype(np.int8)   # what stands there before the call

    def oracle(self):
        d = oracle.PagedT(self.hq, self.hk, self.D, self.page, self.pages, self.table.shape[1], self.window, self.sinks, *self.s_dy, *self.o_dy)
        want = oracle.paged_attention(d, self.q, self.k, self.v, self.table, self.q_start, self.kv_len, self.out)
        return want

    def descs(self, tk, tv):
        return (B.PagedAttentionDesc(self.hq, self.window, self.sinks, B.Dyadic(*self.s_dy), B.Dyadic(*self.o_dy)),
                B.KvCache(tk.data_ptr(), tv.data_ptr(), self.hk, self.D, self.page, self.pages))

    def gathered(self, b):
        """K and V of sequence b as [kv, hk, D]."""
        t = np.arange(self.kv[b])
        page, t = self.table[b][t // self.page].astype(np.int64), t % self.page
        hk, D, P = self.hk, self.D, self.page
        h, c = np.arange(hk)[:, None], np.arange(D)
        base = (page[:, None, None] * hk + h) * (P * D)
        t = t[:, None, None]
        k = self.k[base + t // 16 * (16 * D) + c // 16 * 256 + t % 16 * 16 + c % 16]
        v = self.v[base + t // 64 * (64 * D) + c // 16 * 1024 + t % 16 // 4 * 256 + c % 16 * 16 + t % 64 // 16 * 4 + t % 4]
        return k, v


class Rotary:
    """One call of ibert_rotary_append_i.  skip: rows that have no slot."""

    def __init__(self, seed, rows, hq, hk, D, R, interleaved, page, q_norm=False, k_norm=False, ld=0, skip=(), max_pos=300, std=40.0):
        rng = np.random.default_rng(seed)
        self.rows, self.hq, self.hk, self.D, self.R, self.inter, self.page, self.max_pos = rows, hq, hk, D, R, interleaved, page, max_pos
        self.pages = -(-rows // page) + 2
        heads = hq + 2 * hk
        self.qkv = normal8(rng, std, rows, heads * D + ld)
        if rows:
            self.qkv[0, :D] = 0                     # a head of nothing: its root mean square is zero
            self.qkv[rows - 1, :heads * D] = -128   # the most a head can hold
        self.slots = rng.permutation(self.pages * page)[:rows].astype(np.int32)
        for i in skip:
            self.slots[i] = (-1, self.pages * page, -2 ** 31, 2 ** 31 - 1)[i % 4]
        self.positions = rng.integers(-5, max_pos + 5, rows).astype(np.int32)
        freqs = 10000.0 ** (-np.arange(0, R, 2) / max(R, 1))
        angle = np.arange(max_pos)[:, None] * freqs
        self.cs = np.stack([np.rint(16384 * np.cos(angle)), np.rint(16384 * np.sin(angle))], -1).astype(np.int16)
        gamma = lambda: rng.integers(-16383, 16384, D).astype(np.int32)       # noqa: E731
        self.gq, self.gk = gamma() if q_norm else None, gamma() if k_norm else None
        self.shifts = (int(rng.integers(8, 14)), int(rng.integers(1, 20)))
        after = lambda g, s: dyadic(127 / 4 / 2.0 ** (10 + 13 - s) / 16384) if g is not None else dyadic(0.7 / 16384)     # noqa: E731
        self.q_dy, self.k_dy, self.v_dy = after(self.gq, self.shifts[0]), after(self.gk, self.shifts[1]), dyadic(1.3)
        self.q0 = rng.integers(-127, 128, (rows, hq * D + ld)).astype(np.int8)
        cells = self.pages * page * hk * D
        self.k0, self.v0 = (rng.integers(-127, 128, cells).astype(np.int8) for _ in range(2))

    def oracle(self):
        d = oracle.RotaryT(self.hq, self.hk, self.D, self.page, self.R, int(self.inter), self.max_pos, self.pages, *self.q_dy, *self.k_dy, *self.v_dy, *self.shifts)
        return oracle.rotary_append(d, self.qkv, self.cs if self.R else None, self.positions, self.slots, self.gq, self.gk, self.q0, self.k0, self.v0)

    def descs(self, tk, tv):
        return (B.RotaryDesc(self.hq, self.R, B.ROTARY_INTERLEAVED if self.inter else B.ROTARY_HALF, self.max_pos, B.Dyadic(*self.q_dy), B.Dyadic(*self.k_dy),
                             B.Dyadic(*self.v_dy), *self.shifts),
                B.KvCache(tk.data_ptr(), tv.data_ptr(), self.hk, self.D, self.page, self.pages))


class Pages:
    """One call of ibert_page_tables_i on a consistent state: every page is a sequence's or waits in the ring.  count: how many wait
    (None: enough for all); rows: None: enough for all."""

    def __init__(self, seed, before, after, page, width=None, count=None, rows=None, extra_rows=0, more_pages=3):
        rng = np.random.default_rng(seed)
        self.page = page
        self.before, self.after = np.array(before, np.int32).reshape(-1), np.array(after, np.int32).reshape(-1)
        lb, la = np.maximum(self.before, 0).astype(np.int64), np.maximum(self.after, 0).astype(np.int64)
        had, wants = -(-lb // page), -(-la // page)
        self.width = max(1, int(max(had.max(initial=0), wants.max(initial=0)))) if width is None else width
        held, need = int(had.sum()), int(np.maximum(0, wants - had).sum())
        self.num = max(1, held + (need if count is None else count) + more_pages)
        ids = rng.permutation(self.num)
        self.table = rng.integers(0, self.num, (len(lb), self.width)).astype(np.int32)
        at = 0
        for b, n in enumerate(had):
            self.table[b, :n] = ids[at:at + n]
            at += n
        head = int(rng.integers(0, self.num))
        waiting = (need if count is None else count) + more_pages if count is None else count
        waiting = min(waiting, self.num - held)
        self.ring = rng.integers(0, self.num, self.num).astype(np.int32)
        self.ring[(head + np.arange(waiting)) % self.num] = ids[held:held + waiting]
        self.ring_in = np.array([head, waiting], np.int32)
        self.rows = (int(np.maximum(0, la - lb).sum()) if rows is None else rows) + extra_rows

    def oracle(self):
        return oracle.page_tables(self.before, self.after, self.page, self.ring_in, self.ring, self.table, self.rows)


def mixed_lengths(rng, batch, top):
    """Requests that decode, come, end, shrink and stay."""
    before = rng.integers(0, top, batch)
    kind = rng.integers(0, 5, batch)
    after = np.where(kind == 0, before + 1, np.where(kind == 1, before + rng.integers(0, top, batch), np.where(kind == 2, 0, np.where(kind == 3, before // 2, before))))
    return before, after
