"""CPU checks of the gated block, the products with 4-bit weights and the logits' adjustment: what the entry points refuse, the host helpers,
and the definitions against real arithmetic."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2101_01321_amd import binding as B
import feed_util as U

P = C.c_void_p(1 << 20)              # an address that no refused call touches
Q = C.c_void_p(1 << 40)
R = C.c_void_p(1 << 41)


# ------------------------------------------------------------------------------------------- the definitions
def test_sigmoid_follows_the_real_one():
    # i-exp is off by 2.2e-3 of the octave's top (its polynomial, measured over its 64 arguments below); a weight e moves TOP/(TOP+e) by less than its own share e/TOP's error
    top = 23556
    gap = max(abs(((124 - f) ** 2 + 8180) / top - 2.0 ** (-f / 64)) for f in range(64))
    assert gap < 2.2e-3 and U.SIGMOID[0] == 2 ** 14 and U.SIGMOID[1024] == 2 ** 15 and U.SIGMOID.max() == 2 ** 15
    for d in range(1025):
        real = 1 / (1 + 2.0 ** (-d / 64))
        assert abs(U.SIGMOID[d] / 2 ** 15 - real) <= gap * 2.0 ** -(d // 64) + 0.5 / top + 2.0 ** -16, d
    assert np.all(np.diff(U.SIGMOID) >= 0)


@pytest.mark.parametrize("act", [B.GATE_SILU, B.GATE_GELU])
def test_gated_definition_follows_real_arithmetic(act):
    a = U.Gated(1, 40, 300, 96, act)
    p, y = a.params, a.expected().astype(np.float64)
    S_gate, S_up, S_out = (B.SILU_SCALE if act == B.GATE_SILU else 1 / 200), 1 / 2000, 1 / 16
    real = a.acc * (a.ch.m / 2.0 ** a.ch.s)
    g, u = real[:, :300] * S_gate, np.clip(real[:, 300:], -32767, 32767) * S_up
    if act == B.GATE_SILU:
        want = g / (1 + np.exp(-g))
        # the gate's rounding to a step of ln2/64 moves the sigmoid by at most ln2/128/4, and i-exp by 2.2e-3 of the octave's top in e, of which the sigmoid takes a
        # quarter at most; below d = 64 that is the bound itself
        slack = np.abs(g) * (math.log(2) / 128 / 4 + 2.2e-3 / 1 + 2.0 ** -15) + 2 * S_gate
    else:
        want = 0.5 * g * (1 + np.vectorize(math.erf)(g / math.sqrt(2)))
        # i-GELU's polynomial is off by 1.8e-2 at most over the reals, its constants are rounded down to the scale
        slack = np.full_like(g, 2.2e-2) + np.abs(g) / 200
    bound = slack * np.abs(u) / S_out + (np.abs(want) + slack) * S_up / S_out + 0.51
    assert np.all(np.abs(y - np.clip(want * u / S_out, -127, 127)) <= bound)
    assert p.out_dy.tuple() == U.dyadic((S_gate if act == B.GATE_SILU else S_gate / 4) * S_up / S_out)


def test_gated_definition_at_its_ends():
    p = B.ibert_gate_params_from_scales(B.GATE_SILU, 0, 1 / 32767, 1.0)
    p.out_dy = B.Dyadic(1, 24)
    one = (np.array([1], np.int32).repeat(2), np.array([0], np.int32).repeat(2))
    y = lambda g, u: int(U.gate(np.array([[g]], np.int64), np.array([[u]], np.int64), *one, p)[0, 0])      # noqa: E731
    assert y(U.HIGH, U.HIGH) == 127 and y(U.LOW, U.HIGH) == 0 and y(0, U.HIGH) == 0 and y(U.HIGH, U.LOW) == -127
    assert y(1 << 14, 1 << 10) == 1 and y(1 << 14, -(1 << 10)) == -1 and y(-(1 << 14), 1 << 10) == 0


# ------------------------------------------------------------------------------------------- host helpers
@pytest.mark.parametrize("N,K,group,zeros", [(1, 1, 32, False), (16, 128, 128, True), (17, 129, 64, True), (50, 333, 32, True), (33, 700, 128, False)])
def test_pack_puts_every_weight_in_its_place(N, K, group, zeros):
    w = U.W4(np.random.default_rng(N + K), N, K, group, zeros)
    packed, s, z = w.pack()
    chunks, per = -(-K // 128), 128 // group
    assert packed.size == B.ibert_w4_bytes(N, K) == -(-N // 16) * chunks * 1024 and s.size == B.ibert_w4_scale_bytes(N, K, group) == packed.size // 1024 * 16 * per
    seen = np.zeros((packed.size, 2), int)
    for n in range(N):
        for k in range(K):
            at = (n // 16 * chunks + k // 128) * 1024 + k % 32 // 8 * 256 + n % 16 * 16 + k % 64 // 32 * 8 + k % 8
            high = k % 128 >= 64
            nibble = packed[at] >> 4 if high else packed[at] & 15
            assert (int(nibble) ^ 8) - 8 == w.w[n, k]
            seen[at, int(high)] += 1
            gat = ((n // 16 * chunks + k // 128) * 16 + n % 16) * per + k % 128 // group
            assert s[gat] == w.s[n, k // group] and (z is None or z[gat] == w.z[n, k // group])
    assert seen.max() == 1 and seen.sum() == N * K
    assert all(packed[i] & 15 == 0 for i in np.flatnonzero(seen[:, 0] == 0)) and all(packed[i] >> 4 == 0 for i in np.flatnonzero(seen[:, 1] == 0))


def test_pack_refuses():
    ok = (np.zeros((4, 40), np.int8), np.ones((4, 2), np.uint8))
    B.ibert_w4_pack(*ok, None, 32)
    for w, s, z, group, code in ((ok[0] + 8, ok[1], None, 32, -3), (ok[0] - 9, ok[1], None, 32, -3), (ok[0], ok[1], ok[1].astype(np.int8) + 7, 32, -3)):
        with pytest.raises(B.IbertError) as e:
            B.ibert_w4_pack(w, s, z, group)
        assert e.value.code == code
    for bad in ((0, 40, 32), (4, 0, 32), ((1 << 24) + 1, 40, 32), (4, (1 << 17) + 1, 32)):
        assert B.ibert_w4_bytes(*bad[:2]) == 0 and B.lib().ibert_w4_pack(P, P, None, *bad, P, P, None) == -2
    assert B.ibert_w4_scale_bytes(4, 40, 16) == 0 and B.lib().ibert_w4_pack(P, P, None, 4, 40, 16, P, P, None) == -3
    w, s = ok[0].ctypes.data, ok[1].ctypes.data
    for args in ((None, s, None, P, P, None), (w, None, None, P, P, None), (w, s, None, None, P, None), (w, s, None, P, None, None), (w, s, s, P, P, None)):
        assert B.lib().ibert_w4_pack(*args[:3], 4, 40, 32, *args[3:]) == -1
    with pytest.raises(ValueError):
        B.ibert_w4_pack(np.zeros((4, 40), np.int8), np.ones((4, 1), np.uint8), None, 32)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_weights_from_reals_are_near(group):
    rng = np.random.default_rng(group)
    x = rng.normal(0, 1, (30, 301)) * rng.uniform(0.05, 3, (30, 1)) * np.repeat(rng.uniform(0.2, 1, (30, -(-301 // group))), group, 1)[:, :301]
    x[3] = 0
    x[4, :group] = 0
    w, s, S = B.ibert_w4_from_float(x, group)
    scale = np.repeat(s.astype(np.float64), group, 1)[:, :301] * S[:, None]
    top = np.repeat(np.stack([np.abs(x[:, g:g + group]).max(1) for g in range(0, 301, group)], 1), group, 1)[:, :301]
    # half a step of the group, and where the integer scale was rounded down by half a unit, seven times that half for the values cut off at 7
    assert np.all(np.abs(x - w * scale) <= np.maximum(0.5 * scale, 3.5 * S[:, None]) + 0.5 * S[:, None] + 1e-12 * top)
    assert np.abs(w).max() == 7 and s.max() == 255 and S[3] == 1 and not s[3].any() and s[4, 0] == 0 and s[4, 1] > 0
    for bad in (np.nan, np.inf, -np.inf):
        y = x.copy()
        y[7, 11] = bad
        with pytest.raises(B.IbertError) as e:
            B.ibert_w4_from_float(y, group)
        assert e.value.code == -3
    with pytest.raises(B.IbertError):
        B.ibert_w4_from_float(np.full((1, 5), 1e-308), group)


def test_gate_params_refuse():
    for args in ((2, 1.0, 1.0, 1.0), (-1, 1.0, 1.0, 1.0), (0, 0.0, 0.0, 1.0), (0, 0.0, 1.0, 0.0), (1, 0.0, 1.0, 1.0), (1, -1.0, 1.0, 1.0), (0, 0.0, 1e30, 1e-30)):
        with pytest.raises(B.IbertError) as e:
            B.ibert_gate_params_from_scales(*args)
        assert e.value.code == -3
    assert B.lib().ibert_gate_params_from_scales(0, 0.0, 1.0, 1.0, None) == -1


def test_gelu_gates_reach_where_gelu_is_straight():
    # what a gate can be at most, q_max S_gate, against -q_b S_gate = 2.50, from where on the integer erf is one: a finer scale cuts off gates at which GELU is still curved
    for n in (10, 50, 100, 200, 300, 350, 390, 394, 395):
        p = B.ibert_gate_params_from_scales(B.GATE_GELU, 1 / n, 1 / 2000, 1 / 16).gelu
        assert p.q_max >= -p.q_b and abs(p.q_max / n / (1.55e8 / n ** 3) - 1) < 0.02, n
    for n in (397, 398, 400, 450, 1500, 10000):
        whole = B.ibert_gelu_params_from_scale(1 / n, 1 / (4 * n))
        assert whole.q_max < -whole.q_b, n
        with pytest.raises(B.IbertError) as e:
            B.ibert_gate_params_from_scales(B.GATE_GELU, 1 / n, 1 / 2000, 1 / 16)
        assert e.value.code == -3
        B.ibert_gate_params_from_scales(B.GATE_SILU, 1 / n, 1 / 2000, 1 / 16)      # (not used with SiLU)


def test_logits_row_from_reals():
    p = B.ibert_logits_row_from_reals(0.01, 1.25, 0.5, -0.1, 3)
    assert p.up.tuple() == U.dyadic(0.8) and p.down.tuple() == U.dyadic(1.25) and (p.presence, p.frequency, p.mask) == (50, -10, 3)
    for args in ((0.0, 1.0, 0, 0), (1.0, 0.0, 0, 0), (1.0, -1.0, 0, 0), (1.0, math.inf, 0, 0), (1e-9, 1.0, 3.0, 0), (1e-9, 1.0, 0, 3.0), (1.0, 1.0, math.nan, 0), (1.0, 1e-30, 0, 0)):
        with pytest.raises(B.IbertError) as e:
            B.ibert_logits_row_from_reals(*args)
        assert e.value.code == -3
    assert B.lib().ibert_logits_row_from_reals(1.0, 1.0, 0.0, 0.0, 0, None) == -1


# ------------------------------------------------------------------------------------------- refusals
def gated_desc(**change):
    d = B.GatedDesc(4, 32, 64, 64, 64, 32, B.ibert_gate_params_from_scales(B.GATE_GELU, 1 / 200, 1 / 2000, 1 / 16))
    for k, v in change.items():
        setattr(d, k, v)
    return d


def w4_weights(**change):
    w = B.W4Weights((1 << 40) + 1024, (1 << 41), None, 64)
    for k, v in change.items():
        setattr(w, k, v)
    return w


def i8_gated(d, A=P, W=Q, bias=None, m=R, s=R, c=C.c_void_p(1 << 30)):
    return B.lib().ibert_gemm_i8_gated(None if d is None else C.byref(d), A, W, bias, m, s, c, None)


def w4_gated(d, A=P, g=None, u=None, m=R, s=R, c=C.c_void_p(1 << 30)):
    g, u = w4_weights() if g is None else g, w4_weights() if u is None else u
    return B.lib().ibert_gemm_w4_gated(None if d is None else C.byref(d), A, C.byref(g) if g else None, C.byref(u) if u else None, None, m, s, c, None)


@pytest.mark.parametrize("call", [i8_gated, w4_gated])
def test_gated_refuses(call):
    for change, code in (({"M": -1}, -2), ({"F": -1}, -2), ({"K": 0}, -2), ({"K": -3}, -2), ({"K": (1 << 17) + 1, "lda": 1 << 18, "ldw": 1 << 18}, -2),
                         ({"F": (1 << 24) + 1, "ldc": 1 << 25}, -2), ({"lda": 63}, -2), ({"ldc": 31}, -2)):
        assert call(gated_desc(**change)) == code, change
    d = gated_desc()
    for act in (-1, 2):
        d.gate.activation = act
        assert call(d) == -3
    for field, value in (("q_b", 1), ("q_max", -1), ("q_max", 1 << 30), ("out", B.Dyadic(1, 63)), ("out", B.Dyadic(1, -1))):
        d = gated_desc()
        setattr(d.gate.gelu, field, value)
        assert call(d) == -3, field
        d.gate.activation, d.M = B.GATE_SILU, 0                    # (not used with SiLU)
        assert call(d) == 0
    for s in (-1, 63):
        d = gated_desc()
        d.gate.out_dy = B.Dyadic(1, s)
        assert call(d) == -3
    assert call(None) == -1 and call(gated_desc(), A=None) == -1 and call(gated_desc(), m=None) == -1 and call(gated_desc(), s=None) == -1 and call(gated_desc(), c=None) == -1
    for change in ({"M": 0}, {"F": 0}):
        assert call(gated_desc(**change), A=None, m=None, s=None, c=None) == 0
    assert call(gated_desc(), c=C.c_void_p(P.value + 3 * 64 + 63)) == -2 and call(gated_desc(), c=C.c_void_p(P.value - 3 * 32 - 31)) == -2      # the output over A's last byte, its last over A's first


def test_i8_gated_refuses_its_weights():
    assert i8_gated(gated_desc(ldw=63)) == -2 and i8_gated(gated_desc(), W=None) == -1
    assert i8_gated(gated_desc(), c=C.c_void_p(Q.value + 63 * 64 + 63)) == -2


def test_w4_gated_refuses_its_weights():
    d = gated_desc(ldw=0, M=4)
    for which in ("g", "u"):
        for change, code in (({"group": 16}, -3), ({"group": 0}, -3), ({"group": 256}, -3), ({"w": None}, -1), ({"scales": None}, -1), ({"w": (1 << 40) + 8}, -4),
                             ({"scales": (1 << 41) + 2}, -4), ({"zeros": (1 << 42) + 1}, -4), ({"group": 32}, -3), ({"zeros": 1 << 42}, -3)):
            assert w4_gated(d, **{which: w4_weights(**change)}) == code, (which, change)
        assert w4_gated(d, **{which: False}) == -1
    assert w4_gated(d, c=C.c_void_p((1 << 40) + 1024)) == -2


def w4_desc(**change):
    d = B.W4Desc(4, 32, 64, B.I16, 64, 32, 32, 32767, B.Dyadic(1, 0))
    for k, v in change.items():
        setattr(d, k, v)
    return d


def w4(d, A=P, w=None, m=R, s=R, r=None, c=C.c_void_p(1 << 30)):
    w = w4_weights() if w is None else w
    return B.lib().ibert_gemm_w4_requant(None if d is None else C.byref(d), A, C.byref(w) if w else None, None, m, s, r, c, None)


def test_w4_refuses():
    res = C.c_void_p(1 << 35)
    for change, code in (({"M": -1}, -2), ({"N": -1}, -2), ({"K": 0}, -2), ({"K": (1 << 17) + 1, "lda": 1 << 18}, -2), ({"N": (1 << 24) + 1, "ldc": 1 << 25, "ldr": 1 << 25}, -2),
                         ({"lda": 63}, -2), ({"ldc": 31}, -2), ({"ldr": 31}, -2), ({"out_dtype": 3}, -3), ({"out_dtype": -1}, -3), ({"out_clamp": -1}, -3),
                         ({"out_clamp": 32768}, -3), ({"out_dtype": B.I8, "out_clamp": 128}, -3), ({"residual_dy": B.Dyadic(1, 63)}, -3), ({"residual_dy": B.Dyadic(1, -1)}, -3)):
        assert w4(w4_desc(**change), r=res) == code, change
    assert w4(None) == -1 and w4(w4_desc(), A=None) == -1 and w4(w4_desc(), m=None) == -1 and w4(w4_desc(), s=None) == -1 and w4(w4_desc(), c=None) == -1 and w4(w4_desc(), w=False) == -1
    for change, code in (({"group": 48}, -3), ({"w": None}, -1), ({"scales": None}, -1), ({"w": (1 << 40) + 4}, -4), ({"scales": (1 << 41) + 1}, -4), ({"zeros": (1 << 42) + 2}, -4)):
        assert w4(w4_desc(), w=w4_weights(**change)) == code, change
    for change in ({"M": 0}, {"N": 0}, {"M": 0, "residual_dy": B.Dyadic(1, 99)}):
        assert w4(w4_desc(**change), A=None, m=None, s=None, c=None) == 0
    assert w4(w4_desc(), c=C.c_void_p(P.value + 255)) == -2 and w4(w4_desc(), c=C.c_void_p((1 << 40) + 1024)) == -2 and w4(w4_desc(), r=res, c=res) == -2


def logits(d, x=P, p=R, tok=R, ts=R, os=R, ids=R, vals=R, bs=R, masks=R, y=Q):
    return B.lib().ibert_logits_adjust_i(None if d is None else C.byref(d), x, p, tok, ts, os, ids, vals, bs, masks, y, None)


def logits_desc(**change):
    d = B.LogitsDesc(4, 100, 104, 108, 7, 5, 2, 4)
    for k, v in change.items():
        setattr(d, k, v)
    return d


def test_logits_refuse():
    for change in ({"rows": -1}, {"vocab": -1}, {"vocab": (1 << 26) + 1, "ldx": 1 << 27, "ldy": 1 << 27, "ld_mask": 1 << 23}, {"ldx": 99}, {"ldy": 99}, {"num_tokens": -1},
                   {"num_tokens": 1 << 30}, {"num_biases": -1}, {"num_biases": 1 << 30}, {"num_masks": -1}, {"ld_mask": 3}):
        assert logits(logits_desc(**change)) == -2, change
    assert logits(None) == -1
    for name in ("x", "p", "tok", "ts", "os", "ids", "vals", "bs", "masks", "y"):
        assert logits(logits_desc(), **{name: None}) == -1, name
    assert logits(logits_desc(rows=0), x=None, y=None) == 0 and logits(logits_desc(vocab=0, ld_mask=0), x=None, y=None) == 0
    # y over x: not with another leading dimension, not shifted
    assert logits(logits_desc(), y=P) == -2 and logits(logits_desc(ldy=104), y=C.c_void_p(P.value + 4)) == -2 and logits(logits_desc(ldy=104), y=C.c_void_p(P.value - 4)) == -2
    assert logits(logits_desc(), y=C.c_void_p(P.value + 4 * (3 * 104 + 99))) == -2


def test_leading_dimensions_beyond_any_memory_do_not_wrap():
    # rows 2^62 apart: their extent passes 64 bits; what stands between two rows of the one is not taken for free of the other
    d = w4_desc(lda=1 << 62, M=5)
    assert w4(d, c=C.c_void_p(P.value + 64)) == -2
    assert i8_gated(gated_desc(ldw=1 << 62), c=C.c_void_p(Q.value + 64)) == -2 and i8_gated(gated_desc(lda=1 << 62), c=C.c_void_p(P.value + 64)) == -2
    assert logits(logits_desc(ldx=1 << 62), y=C.c_void_p(P.value + 400)) == -2


def test_structs_have_the_header_s_sizes():
    # ctypes and the C compiler agree on natural alignment; the arrays a program makes itself have 28 bytes a row
    assert C.sizeof(B.LogitsRow) == 28 and C.sizeof(B.GateParams) == 4 + 24 + 8 and C.sizeof(B.W4Weights) == 32 and C.sizeof(B.W4Desc) == 56
    assert C.sizeof(B.GatedDesc) == 16 + 24 + 40 and C.sizeof(B.LogitsDesc) == 40


def test_logits_by_rows_are_those_token_by_token():
    for seed, (lens, vocab, blens, masks, ld) in enumerate([([3], 1, [1], 1, (0, 0, 0)), ([0, 500, 77], 333, [9, 0, 300], 3, (3, 5, 2)), ([50, 60, 70, 80], 400, [20, 30, 10, 5], 0, (0, 0, 0))]):
        c = U.Logits(seed, lens, vocab, blens, masks, ld)
        assert np.array_equal(U.logits_by_rows(c), c.expected())
        if len(lens) == 4:
            c.start[:], c.made[:], c.bstart[:] = (-7, 10 ** 9, 100, U.LOW, U.HIGH), (U.LOW, 10 ** 8, 120, 100), (30, 20, -1, 10 ** 9, 40)
            c.params[0, 1], c.params[1, 3], c.params[2, 1], c.params[3, 1] = 63, -1, U.HIGH, U.LOW
            assert np.array_equal(U.logits_by_rows(c, c.y0), c.expected(c.y0))
