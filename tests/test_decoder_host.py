"""CPU checks of the decoder attention: what the entry points refuse, the host helpers against closed forms, and the oracle of
the three operators against real arithmetic and against its own invariants."""
import ctypes as C
import math

import numpy as np
import pytest

import oracle
from oracle import params as P
from paper_2101_01321_amd import binding as B
import decoder_util as U


# ------------------------------------------------------------------------------------------- the oracle
def test_weight_follows_the_real_exponential():
    # Eq. 13's constants at S = ln2/64: floor(b/S), floor(c/(a S^2)); the largest weight fits 15 bits
    S = math.log(2) / 64
    assert (math.floor(1.353 / S), math.floor(0.344 / (0.3585 * S * S))) == (124, 8180)
    top = 124 ** 2 + 8180
    assert oracle.weight(0) == top < 2 ** 15
    # the polynomial's own distance from 2^(-f/64), measured exactly over its 64 arguments; it halves with each octave, and the
    # rounding adds half a unit
    gap = max(abs(((124 - f) ** 2 + 8180) / top - 2.0 ** (-f / 64)) for f in range(64))
    assert gap < 2.2e-3
    for d in range(0, 1100):
        w = oracle.weight(d)
        assert abs(w / top - 2.0 ** (-d / 64)) <= gap * 2.0 ** (-(d // 64)) + 0.5 / top, d
        assert d == 0 or w <= oracle.weight(d - 1)
    assert oracle.weight(1023) in (0, 1) and oracle.weight(1024) == 0 and oracle.weight(1 << 40) == 0


@pytest.mark.parametrize("hq,hk,D,n,kv,window,sinks", [(4, 2, 64, [1, 3], [70, 200], 0, 0), (2, 2, 128, [5], [131], 0, 0), (6, 1, 64, [4, 1], [90, 300], 40, 3)])
def test_attention_oracle_follows_real_softmax(hq, hk, D, n, kv, window, sinks):
    a = U.Attention(1, hq, hk, D, 64, n, kv, window, sinks, std=25.0)
    got = a.oracle()
    scale = (6.0 / 127) ** 2 / math.sqrt(D)
    for b in range(a.batch):
        k, v = a.gathered(b)
        for i in range(n[b]):
            pos = kv[b] - n[b] + i
            j = np.arange(pos + 1)
            see = j[(j > pos - window) | (j < sinks)] if window else j
            for h in range(hq):
                x = a.q[a.q_start[b] + i, h * D:(h + 1) * D].astype(np.float64)
                s = k[see, h // (hq // hk)].astype(np.float64) @ x * scale
                p = np.exp(s - s.max())
                vv = v[see, h // (hq // hk)].astype(np.float64)
                real = (p[:, None] * vv).sum(0) / p.sum()
                # a weight is off by half a step of ln2/64 and by the polynomial (2.2e-3 of the octave's top, which is at most twice the
                # weight), relative to itself, and by half a unit of 1/23556; a mean moves by at most that share of the values' span
                eps = (2 ** (0.5 / 64) - 1) + 2 * 2.2e-3
                off = (eps + see.size * 0.5 / 23556 / p.sum()) * (vv.max(0) - vv.min(0))
                y = got[a.q_start[b] + i, h * D:(h + 1) * D]
                # (a third of the value's scale, two roundings, and floor(2^48 / W): at least 16 bits of it)
                assert np.all(np.abs(y - np.clip(3 * real, -127, 127)) <= 3 * off + 0.5 + 3 * 127 * 2.0 ** -16 + 1e-3)


def test_attention_oracle_by_hand():
    # one key: the value itself; a row in front of the first key: nothing; equal keys: the mean; a sink beside a window of one
    a = U.Attention(2, 1, 1, 64, 64, [3], [2], out_scale=1.0)
    got, (k, v) = a.oracle(), a.gathered(0)
    assert np.all(got[0] == 0) and np.array_equal(got[1], v[0, 0])
    a = U.Attention(3, 1, 1, 64, 64, [1], [40], out_scale=1.0)
    a.q[:] = 0
    v = a.gathered(0)[1][:, 0].astype(np.int64)
    # the mean v.sum / 40 with 16 bits, through floor(2^48 / W): off by less than 2^-15, which decides nothing but ties
    mean = v.sum(0) / 40
    clear = np.abs(mean - np.floor(mean) - 0.5) > 1e-3
    assert np.array_equal(a.oracle()[0][clear], np.rint(mean).astype(np.int8)[clear]) and clear.sum() > 30
    a = U.Attention(4, 1, 1, 64, 64, [1], [40], window=1, sinks=1, out_scale=1.0)
    a.q[:] = 0
    v = a.gathered(0)[1][:, 0].astype(np.int64)
    mean = (v[0] + v[39]) / 2
    clear = mean == np.rint(mean)
    assert np.array_equal(a.oracle()[0][clear], mean[clear].astype(np.int8))


@pytest.mark.parametrize("D,R,inter", [(64, 64, False), (64, 32, True), (128, 128, True), (128, 16, False), (64, 0, False)])
def test_rotary_oracle_follows_real_rotation(D, R, inter):
    a = U.Rotary(5, 9, 4, 2, D, R, inter, 64, max_pos=5000, std=30.0)
    q, k, v = a.oracle()
    pos = np.clip(a.positions, 0, a.max_pos - 1)
    theta = 10000.0 ** (-np.arange(0, R, 2) / max(R, 1))
    for t in range(a.rows):
        for h in range(4):
            x = a.qkv[t, h * D:(h + 1) * D].astype(np.float64)
            z = x[:R][0::2] + 1j * x[:R][1::2] if inter else x[:R // 2] + 1j * x[R // 2:R]
            z = z * np.exp(1j * pos[t] * theta)
            y = x.copy()
            y[:R] = np.stack([z.real, z.imag], -1).reshape(-1) if inter else np.concatenate([z.real, z.imag])
            # table entries are off by half of 2^-14, two of them at most 128 each; then one rounding
            want = np.clip(0.7 * y, -127, 127)
            assert np.all(np.abs(q[t, h * D:(h + 1) * D] - want) <= 0.5 + 0.7 * 256 * 2.0 ** -15 + 1e-6)


def test_head_norm_oracle_follows_real_norm():
    D, rng = 128, np.random.default_rng(6)
    a = U.Rotary(6, 7, 2, 2, D, 0, False, 64, q_norm=True)
    gamma = rng.normal(1.0, 0.2, D)
    a.gq, shift = B.ibert_head_norm_from_float(gamma, 2.0 ** -12)
    a.shifts = (shift, 1)
    a.q_dy = U.dyadic(127 / 4 / 4096 / 16384)
    q = a.oracle()[0]
    for t in range(a.rows):
        for h in range(2):
            x = a.qkv[t, h * D:(h + 1) * D].astype(np.float64)
            rms = math.sqrt((x * x).mean())
            if rms == 0:
                assert np.all(q[t, h * D:(h + 1) * D] == 0)
                continue
            y = x / rms * gamma
            # sigma with 8 fractional bits is at most 1 / (256 rms) low, floor(2^30 / sigma) at most sigma / 2^30; n loses up to 2^-10, gamma is off
            # by 2^-(shift-9) S_out, u by half of 2^-12; and the last rounding
            rel = 1 / (256 * rms - 1) + 256 * rms / 2.0 ** 30
            off = np.abs(y) * rel + np.abs(gamma) * 2.0 ** -10 + np.abs(x / rms) * 2.0 ** (9 - shift) * 2.0 ** -12 + 2.0 ** -13
            want = np.clip(y * 127 / 4, -127, 127)
            assert np.all(np.abs(q[t, h * D:(h + 1) * D] - want) <= 0.5 + 127 / 4 * off)


def test_pages_are_never_shared_nor_lost():
    rng = np.random.default_rng(7)
    batch, page, width, num, rows = 13, 64, 9, 60, 500
    lens, table = np.zeros(batch, np.int32), np.zeros((batch, width), np.int32)
    ring, state = rng.permutation(num).astype(np.int32), np.array([17, num], np.int32)
    ring = np.roll(ring, 17)
    refused = 0
    for _ in range(200):
        kind = rng.integers(0, 4, batch)
        after = np.where(kind == 0, lens + 1, np.where(kind == 1, lens + rng.integers(0, 150, batch), np.where(kind == 2, lens - rng.integers(0, 100, batch), 0 * (rng.random() < 0.2) + lens)))
        o = oracle.page_tables(lens, after, page, state, ring, table, rows)
        table, ring, state = o["table"], o["ring"], o["ring_out"]
        refused += int(state[2])
        held = [table[b, p] for b in range(batch) for p in range(-(-int(o["kv_len"][b]) // page))]
        free = [ring[(state[0] + i) % num] for i in range(state[1])]
        assert sorted(held + free) == list(range(num))
        real = o["slots"][:o["q_start"][-1]]
        assert len(set(real.tolist())) == real.size and np.all(o["slots"][real.size:] == -1)
        lens = o["kv_len"]
    assert refused > 20


# ------------------------------------------------------------------------------------------- host helpers
def test_rotary_helpers_follow_their_formulas():
    R = 64
    plain = 10000.0 ** (-np.arange(0, R, 2) / R)
    f = lambda kind, **kw: B.ibert_rotary_freqs(B.RotaryScaling(10000.0, kw.get("factor", 4.0), 4096.0, 1.0, 32.0, kind), kw.get("R", R))   # noqa: E731
    assert np.allclose(f(B.ROPE_NONE, factor=0.0), plain, rtol=1e-14)
    assert np.allclose(f(B.ROPE_LINEAR), plain / 4, rtol=1e-14)
    base = f(B.ROPE_BASE)
    assert math.isclose(base[0], 1.0) and math.isclose(base[-1], plain[-1] / 4, rel_tol=1e-12)     # the slowest pair is stretched by the factor
    ramp = f(B.ROPE_RAMP)
    turns = plain * 4096 / (2 * math.pi)
    assert np.array_equal(ramp[turns >= 32], f(B.ROPE_NONE)[turns >= 32]) and np.allclose(ramp[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)
    assert np.all(ramp <= plain * (1 + 1e-14)) and np.all(ramp >= plain / 4 * (1 - 1e-14)) and np.any((ramp < plain * 0.99) & (ramp > plain / 4 * 1.01))
    assert np.allclose(f(B.ROPE_BASE, factor=1.0), plain, rtol=1e-14)
    t = B.ibert_rotary_table_from_freqs(plain, 131072)
    assert t.shape == (131072, R // 2, 2) and t.dtype == np.int16 and tuple(t[0, 5]) == (16384, 0)
    for p in (1, 4097, 131071):
        assert np.array_equal(t[p, :, 0], np.rint(16384 * np.cos(p * plain))) and np.array_equal(t[p, :, 1], np.rint(16384 * np.sin(p * plain)))
    assert B.ibert_rotary_table_from_freqs(plain[:0], 7).shape == (7, 0, 2)


def test_head_norm_and_attention_helpers_follow_their_formulas():
    gamma = np.random.default_rng(8).normal(1, 0.3, 128)
    g, s = B.ibert_head_norm_from_float(gamma, 2.0 ** -12)
    assert np.array_equal(g, np.rint(gamma * 4096 * 2.0 ** (s - 10))) and np.abs(g).max() < 16384
    assert s == 30 or np.abs(np.rint(gamma * 4096 * 2.0 ** (s - 9))).max() >= 16384
    d = B.ibert_paged_attention_from_scales(0.04, 0.05, 0.03, 0.02, 128, 32, 1024, 4)
    assert d.scores_dy.tuple() == P.dyadic_from_double(0.04 * 0.05 / math.sqrt(128.0) * 64.0 / math.log(2)) and d.out_dy.tuple() == P.dyadic_from_double(0.03 / 0.02 / 65536)
    assert (d.heads_q, d.window, d.sinks) == (32, 1024, 4)
    d = B.ibert_paged_attention_from_scales(1e-9, 1e-9, 1, 1, 64, 4)
    assert (d.scores_dy.m, d.scores_dy.s) == (0, 62)


@pytest.mark.parametrize("call", [
    lambda: B.ibert_rotary_freqs(B.RotaryScaling(0.0, 1, 1, 0, 1, 0), 64), lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, 0.5, 1, 0, 1, B.ROPE_LINEAR), 64),
    lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, 2, 1, 0, 1, 4), 64), lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, 2, 4096, 4, 4, B.ROPE_RAMP), 64),
    lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, 2, 0, 1, 4, B.ROPE_RAMP), 64), lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, 2, 1, 0, 1, B.ROPE_BASE), 2),
    lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, float("nan"), 1, 0, 1, B.ROPE_LINEAR), 64), lambda: B.ibert_rotary_freqs(B.RotaryScaling(1e4, 1, 1, 0, 1, 0), 7),
    lambda: B.ibert_rotary_table_from_freqs(np.array([np.inf]), 4), lambda: B.ibert_head_norm_from_float(np.ones(64), 0.0), lambda: B.ibert_head_norm_from_float(np.full(64, 1e9), 1e-9),
    lambda: B.ibert_paged_attention_from_scales(40.0, 40.0, 1, 1, 64, 4), lambda: B.ibert_paged_attention_from_scales(1, -1, 1, 1, 64, 4)])
def test_helpers_refuse(call):
    with pytest.raises(B.IbertError):
        call()


# ------------------------------------------------------------------------------------------- refusals
DUMMY = 4096           # a non-NULL address that nothing reads: validation fails before


def cache(**kw):
    c = B.KvCache(DUMMY, DUMMY, 2, 64, 64, 10)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(heads_kv=0), -2), (dict(heads_kv=1025), -2), (dict(head_dim=96), -7), (dict(page_size=32), -2), (dict(page_size=96), -2), (dict(num_pages=0), -2),
              (dict(num_pages=1 << 25), -2)]


def test_cache_bytes():
    assert B.ibert_kv_cache_bytes(cache()) == 10 * 64 * 2 * 64
    assert B.ibert_kv_cache_bytes(cache(num_pages=(1 << 25) - 1, head_dim=128, heads_kv=1024)) == ((1 << 25) - 1) * 64 * 1024 * 128
    for kw, _ in BAD_CACHES:
        assert B.ibert_kv_cache_bytes(cache(**kw)) == 0


def test_page_tables_refuse():
    def call(batch=3, page=64, num=10, width=4, rows=5, **kw):
        p = {k: 4096 + 256 * i for i, k in enumerate(("before", "after", "ring_in", "ring", "ring_out", "table", "q_start", "kv_len", "slots", "positions"))}
        p.update(kw)
        return B.lib().ibert_page_tables_i(p["before"], p["after"], batch, page, num, p["ring_in"], p["ring"], p["ring_out"], p["table"], width, rows, p["q_start"],
                                           p["kv_len"], p["slots"], p["positions"], None)
    for kw in (dict(batch=-1), dict(batch=8193), dict(page=48), dict(page=32), dict(num=0), dict(width=0), dict(rows=-1), dict(num=1 << 25), dict(width=1 << 25),
               dict(batch=8192, width=1 << 18), dict(ring_out=4096 + 512), dict(kv_len=4096), dict(kv_len=4096 + 256)):
        assert call(**kw) == -2, kw
    for name in ("before", "after", "ring_in", "ring", "ring_out", "table", "q_start", "kv_len", "slots", "positions"):
        assert call(**{name: None}) == -1, name


def test_rotary_refuses():
    def call(c=None, rows=3, ld=8 * 64, ld_q=4 * 64, desc=None, **kw):
        d = B.RotaryDesc(4, 64, 0, 100, B.Dyadic(1, 0), B.Dyadic(1, 0), B.Dyadic(1, 0), 5, 5)
        for k, v in (desc or {}).items():
            setattr(d, k, v)
        p = dict(qkv=DUMMY, table=DUMMY, positions=DUMMY, slots=DUMMY, gq=None, gk=None, q=DUMMY)
        p.update(kw)
        return B.lib().ibert_rotary_append_i(C.byref(d), C.byref(c or cache()), p["qkv"], ld, p["table"], p["positions"], p["slots"], p["gq"], p["gk"], rows, p["q"], ld_q, None)
    for kw, rc in BAD_CACHES:
        assert call(c=cache(**kw)) == rc, kw
    for kw in (dict(rows=-1), dict(ld=8 * 64 - 16), dict(ld_q=4 * 64 - 16), dict(desc=dict(heads_q=0)), dict(desc=dict(heads_q=5)), dict(rows=1 << 62), dict(rows=1 << 31)):
        assert call(**kw) == -2, kw
    for kw in (dict(desc=dict(rot_dim=-16)), dict(desc=dict(rot_dim=8)), dict(desc=dict(rot_dim=80)), dict(desc=dict(layout=2)), dict(desc=dict(max_pos=0)),
               dict(desc=dict(q_dy=B.Dyadic(1, 63))), dict(desc=dict(k_dy=B.Dyadic(1, -1))), dict(desc=dict(v_dy=B.Dyadic(1, 63))),
               dict(gq=DUMMY, desc=dict(q_norm_shift=0)), dict(gk=DUMMY, desc=dict(k_norm_shift=31))):
        assert call(**kw) == -3, kw
    for name in ("qkv", "table", "positions", "slots", "q"):
        assert call(**{name: None}) == -1, name
    assert call(c=cache(k=None)) == -1 and call(c=cache(v=None)) == -1
    for kw in (dict(qkv=DUMMY + 8), dict(q=DUMMY + 8), dict(table=DUMMY + 4), dict(gq=DUMMY + 8), dict(gk=DUMMY + 4), dict(ld=8 * 64 + 8), dict(ld_q=4 * 64 + 8), dict(c=cache(k=DUMMY + 8)), dict(c=cache(v=DUMMY + 1))):
        assert call(**kw) == -4, kw
    assert call(rows=0, qkv=None, q=None, slots=None) == 0


def test_paged_attention_refuses():
    L = B.lib()

    def call(c=None, ld_q=256, width=4, batch=2, rows=2, max_q=1, max_kv=200, ld_out=256, ws=0, desc=None, **kw):
        d = B.PagedAttentionDesc(4, 0, 0, B.Dyadic(1, 30), B.Dyadic(1, 16))
        for k, v in (desc or {}).items():
            setattr(d, k, v)
        p = dict(q=DUMMY, table=DUMMY, start=DUMMY, kv=DUMMY, out=DUMMY, workspace=None)
        p.update(kw)
        return L.ibert_paged_attention_i(C.byref(d), C.byref(c or cache()), p["q"], ld_q, p["table"], width, p["start"], p["kv"], batch, rows, max_q, max_kv, p["out"], ld_out,
                                         p["workspace"], ws, None)
    for kw, rc in BAD_CACHES:
        assert call(c=cache(**kw)) == rc, kw
    for kw in (dict(batch=-1), dict(batch=65536), dict(rows=-1), dict(max_q=0), dict(max_q=64 * 65535 // 2 + 1), dict(max_kv=-1), dict(ld_q=240), dict(ld_out=255), dict(width=0), dict(desc=dict(heads_q=3)),
               dict(desc=dict(heads_q=0)), dict(start=None, rows=1)):
        assert call(**kw) == -2, kw
    for kw in (dict(max_kv=131073), dict(desc=dict(window=-1)), dict(desc=dict(sinks=-1)), dict(desc=dict(scores_dy=B.Dyadic(-1, 30))), dict(desc=dict(scores_dy=B.Dyadic(1, 23))),
               dict(desc=dict(scores_dy=B.Dyadic(1, 63))), dict(desc=dict(out_dy=B.Dyadic(1, 63)))):
        assert call(**kw) == -3, kw
    for name in ("q", "table", "kv", "out"):
        assert call(**{name: None}) == -1, name
    assert call(c=cache(k=None)) == -1 and call(c=cache(v=None)) == -1
    for kw in (dict(q=DUMMY + 8), dict(ld_q=264), dict(out=DUMMY + 2), dict(ld_out=258), dict(c=cache(k=DUMMY + 8)), dict(c=cache(v=DUMMY + 8))):
        assert call(**kw) == -4, kw
    assert call(batch=0, q=None, out=None) == 0 and call(rows=0, q=None, out=None) == 0
    d = B.PagedAttentionDesc(4, 0, 0, B.Dyadic(1, 30), B.Dyadic(1, 16))
    need = B.ibert_paged_attention_workspace_bytes(d, cache(num_pages=100000, head_dim=128), 1, 1, 1, 131072)
    if need:
        big = cache(num_pages=100000, head_dim=128)
        for kw in (dict(), dict(workspace=DUMMY, ws=need - 1), dict(workspace=DUMMY + 16, ws=need)):
            assert call(c=big, batch=1, rows=1, width=4096, max_kv=131072, ld_q=512, ld_out=512, **kw) == -5, kw
    assert B.ibert_paged_attention_workspace_bytes(d, cache(), 1, 1, 0, 100) == 0


def test_single_rows_among_prompts_ask_for_the_room_of_single_rows():
    d = B.PagedAttentionDesc(32, 0, 0, B.Dyadic(1, 30), B.Dyadic(1, 16))
    c = cache(heads_kv=8, num_pages=100000, head_dim=128)

    def need(batch, rows, max_q, max_kv):
        return B.ibert_paged_attention_workspace_bytes(d, c, batch, rows, max_q, max_kv)
    singles = need(3, 3, 1, 60000)
    assert singles > 0
    assert need(3, 1026, 1024, 60000) == singles                       # one prompt, two single rows
    assert need(3, 3 * 1024, 1024, 60000) == 0                         # three prompts
    assert need(2, 41, 40, 500) == need(2, 80, 40, 500) == 0           # short ones
    assert B.lib().ibert_paged_attention_i(C.byref(d), C.byref(c), DUMMY, 4096, DUMMY, 1000, DUMMY, DUMMY, 3, 1026, 1024, 60000, DUMMY, 4096, None, 0, None) == -5


def test_page_tables_refuse_what_overlaps():
    # every written array with every other: the same address, and the last word of one on the first of the other
    batch, num, width, rows = 3, 10, 4, 5
    words = dict(ring=num, ring_out=3, table=batch * width, q_start=batch + 1, kv_len=batch, slots=rows, positions=rows, before=batch, after=batch, ring_in=2)
    written = ("ring", "ring_out", "table", "q_start", "kv_len", "slots", "positions")

    def call(batch=batch, rows=rows, **kw):
        p = {k: 1 << 20 | 4096 * i for i, k in enumerate(words)}
        p.update(kw)
        return B.lib().ibert_page_tables_i(p["before"], p["after"], batch, 64, num, p["ring_in"], p["ring"], p["ring_out"], p["table"], width, rows, p["q_start"], p["kv_len"],
                                           p["slots"], p["positions"], None)
    for w in written:
        for o in words:
            if o != w:
                for at in (0, 4 * (words[o] - 1), -4 * (words[w] - 1)):
                    assert call(**{o: 1 << 24, w: (1 << 24) + at}) == -2, (w, o, at)


@pytest.mark.parametrize("first", ["B.ibert_rotary_table_from_freqs(np.ones(4), 3)", "B.lib()", "import torch"])
def test_one_hip_runtime_whatever_is_called_first(first):
    # a process with torch's runtime and the system's beside it has no device for the second of them
    import os
    import subprocess
    import sys
    code = ("import numpy as np\nfrom paper_2101_01321_amd import binding as B\n%s\nimport torch\nB.lib()\n"
            "print(len({line.split()[-1] for line in open('/proc/self/maps') if 'libamdhip64' in line}))" % first)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.run([sys.executable, "-c", code], cwd=root, check=True, capture_output=True, text=True).stdout.split() == ["1"]


@pytest.mark.parametrize("hq,hk,D,batch,rows,max_q,max_kv", [(4, 2, 128, 1, 1, 1, 131072), (12, 12, 64, 1, 1, 1, 4000), (32, 8, 128, 1, 4, 4, 20000), (32, 8, 128, 3, 1026, 1024, 60000)])
def test_a_workspace_that_does_not_do_is_refused(hq, hk, D, batch, rows, max_q, max_kv):
    # one row and a few on many keys, and single rows beside a prompt: without one, a byte short, off its alignment
    d = B.PagedAttentionDesc(hq, 0, 0, B.Dyadic(1, 30), B.Dyadic(1, 16))
    c = cache(heads_kv=hk, num_pages=100000, head_dim=D)
    need = B.ibert_paged_attention_workspace_bytes(d, c, batch, rows, max_q, max_kv)
    assert need > 0
    for at, size in ((None, 0), (None, need), (DUMMY, need - 1), (DUMMY, 0), (DUMMY + 16, need), (DUMMY + 128, need + 256)):
        assert B.lib().ibert_paged_attention_i(C.byref(d), C.byref(c), DUMMY, hq * D, DUMMY, 4096, DUMMY, DUMMY, batch, rows, max_q, max_kv, DUMMY, hq * D, at, size, None) == -5, (at, size)


@pytest.mark.parametrize("scaling,rot_dim", [(B.RotaryScaling(1e300, 1e10, 1, 0, 1, B.ROPE_BASE), 64), (B.RotaryScaling(1e4, 1e200, 1, 0, 1, B.ROPE_BASE), 4), (B.RotaryScaling(5e-324, 1, 1, 0, 1, B.ROPE_NONE), 4096)])
def test_frequencies_that_binary64_does_not_hold_are_refused(scaling, rot_dim):
    # a base of infinity would give 0 for every pair but the first, where the real ones are 1e-10 and less; a base near 0 frequencies of infinity
    with pytest.raises(B.IbertError) as e:
        B.ibert_rotary_freqs(scaling, rot_dim)
    assert e.value.code == -3


def test_a_table_of_angles_that_binary64_does_not_hold_is_refused():
    with pytest.raises(B.IbertError) as e:
        B.ibert_rotary_table_from_freqs(np.array([1.0, 1e308]), 100)
    assert e.value.code == -3
    assert tuple(B.ibert_rotary_table_from_freqs(np.array([1e308]), 1)[0, 0]) == (16384, 0)         # position 0 alone has an angle
