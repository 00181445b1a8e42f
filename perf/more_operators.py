"""The operators around the decoder's attention on cases that can be timed: gated feed-forward products, products with 4-bit
weights and group scales, and what is done to the logits of the vocabulary before Softmax.

Everything is integer and exact.  With `own` false the operators run in their plain form, elementary torch operations (sums of
products in binary64, which holds them exactly); with `own` true they are the library's entry points.

4-bit weights of an [N, K] matrix stand in the order in which the matrix unit takes its operands, N in tiles of 16 and K in chunks
of 128, padded to whole ones:
  w[n / 16][k / 128][k % 32 / 8][n % 16][k % 64 / 32][k % 8], a byte: k % 128 < 64 in its low four bits, k + 64 in the high ones
  scales and zeros: [n / 16][k / 128][n % 16][k % 128 / group]
"""
import math

import numpy as np
import torch

own = False

SILU, GELU = 0, 1
LN2 = math.log(2)
Q_B, Q_C = 124, 8180          # i-exp's constants floor(b/S), floor(c/(a S^2)) at S = ln2/64
TOP = Q_B * Q_B + Q_C         # its value at 0
LOW = -2 ** 31


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the block of a Base-wide decoder for one new token: pure latency
        {"name": "gated_t1_h768", "kind": "gated", "tokens": 1, "hidden": 768, "ffn": 2048, "act": "gelu"},
        # a few requests that decode, and a width that is 8/3 of the hidden size and no multiple of anything
        {"name": "gated_t7_h1024_odd", "kind": "gated", "tokens": 7, "hidden": 1024, "ffn": 2730, "act": "silu"},
        # packed prompts of uneven lengths in a Large-wide decoder
        {"name": "gated_t2741_h1024", "kind": "gated", "tokens": 2741, "hidden": 1024, "ffn": 4096, "act": "gelu"},
        # a large prefill step
        {"name": "gated_t8192_h4096", "kind": "gated", "tokens": 8192, "hidden": 4096, "ffn": 12288, "act": "silu"},
        # the attention's output projection for one new token: pure latency
        {"name": "w4_t1_h768", "kind": "w4", "tokens": 1, "n": 768, "hidden": 768, "group": 64, "zeros": False, "out": "i16"},
        # the down projection behind an odd width, with zero points, small groups
        {"name": "w4_t5_k2730_zeros", "kind": "w4", "tokens": 5, "n": 1024, "hidden": 2730, "group": 32, "zeros": True, "out": "i16"},
        # the vocabulary head of a small batch
        {"name": "w4_t16_vocabulary", "kind": "w4", "tokens": 16, "n": 50265, "hidden": 1024, "group": 128, "zeros": False, "out": "i32"},
        # the down projection of a serving batch in full swing
        {"name": "w4_t64_k12288", "kind": "w4", "tokens": 64, "n": 4096, "hidden": 12288, "group": 128, "zeros": False, "out": "i16"},
        # gate and up projection of one new token in a wide decoder: its weights are all there is to read
        {"name": "w4_gated_t1_h4096", "kind": "w4_gated", "tokens": 1, "hidden": 4096, "ffn": 12288, "group": 128, "zeros": False, "act": "silu"},
        # a small batch, zero points, an odd width
        {"name": "w4_gated_t33_odd", "kind": "w4_gated", "tokens": 33, "hidden": 1024, "ffn": 2730, "group": 64, "zeros": True, "act": "gelu"},
        # one short chat: penalties and a handful of biases, no grammar
        {"name": "logits_b1", "kind": "logits", "rows": 1, "vocab": 50265, "tokens": 77, "biases": 5, "masks": 0},
        # a serving batch: long histories, half of the requests under one of a few grammars
        {"name": "logits_b64_masks", "kind": "logits", "rows": 64, "vocab": 128000, "tokens": 8191, "biases": 300, "masks": 5},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["gated", "w4", "w4_gated", "logits"], [4, 5, 3, 3])[0]
    if kind == "logits":
        rows = _log_int(rng, 1, 256)
        return {"kind": kind, "rows": rows, "vocab": _log_int(rng, 1000, min(160000, 8192000 // rows)), "tokens": _log_int(rng, 1, 8191),
                "biases": rng.choice([0, _log_int(rng, 1, 300)]), "masks": rng.choice([0, 1, rng.randint(2, 20)])}
    hidden = 128 * _log_int(rng, 2, 32) if rng.random() < 0.7 else _log_int(rng, 200, 4096)
    ffn = _log_int(rng, hidden, 3 * hidden) if rng.random() < 0.4 else 64 * _log_int(rng, max(1, hidden // 64), 3 * hidden // 64)
    if kind == "gated":
        top = max(1, min(8192, 8192 * 4096 * 12288 // (hidden * ffn)))
        return {"kind": kind, "tokens": _log_int(rng, 1, top), "hidden": hidden, "ffn": ffn, "act": rng.choice(["gelu", "silu"])}
    tokens, group, zeros = _log_int(rng, 1, 256), rng.choice([32, 64, 128]), rng.random() < 0.4
    if kind == "w4_gated":
        return {"kind": kind, "tokens": tokens, "hidden": hidden, "ffn": ffn, "group": group, "zeros": zeros, "act": rng.choice(["gelu", "silu"])}
    n, k = rng.choice([(hidden, ffn), (ffn, hidden), (hidden, hidden), (3 * hidden // 2, hidden), (_log_int(rng, 8000, 60000), min(hidden, 2048))])
    return {"kind": kind, "tokens": tokens, "n": n, "hidden": k, "group": group, "zeros": zeros, "out": rng.choice(["i8", "i16", "i16", "i32"])}


# ---------------------------------------------------------------------------------------------- inputs
def _dyadic(real):
    """(m, s) with real ~ m / 2^s and m of 31 bits."""
    f, e = math.frexp(real)
    m = round(f * 2 ** 31)
    return (m >> 1, 30 - e) if m == 1 << 31 else (m, 31 - e)


def _normal8(gen, std, *shape):
    return (torch.randn(shape, device="cuda", generator=gen) * std).round_().clamp_(-127, 127).to(torch.int8)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda", dtype)


def _channels(rng, n, acc_std, out_std):
    """Multipliers and shifts of n channels that bring sums of deviation acc_std to about out_std."""
    pairs = [_dyadic(out_std / acc_std * f) for f in rng.uniform(0.7, 1.4, n)]
    return _dev(np.array([p[0] for p in pairs])), _dev(np.array([p[1] for p in pairs]))


def _gelu_constants(S_in, S_out):
    """i-GELU's constants at an input scale, its results at scale S_out."""
    a, b, S = -0.2888, -1.769, S_in / math.sqrt(2)
    q_b, S_erf = math.floor(b / S), a * S * S
    q_c = math.floor(1 / S_erf)
    q_max = (2 ** 31 - 1) // (max(-q_c, abs(q_b * q_b + q_c)) - q_c)
    m, s = _dyadic(-S_in * S_erf / 2 / S_out)
    return {"q_b": q_b, "q_c": q_c, "q_1": q_c, "q_max": q_max, "m": -m, "s": s}


def _gate(case, rng, ffn, acc_std):
    """The constants of a gated block: gates of deviation 1.6, ups in 16 bits."""
    gelu = _gelu_constants(1 / 200, 1 / 800)
    gate_std = 1.6 * 200 if case["act"] == "gelu" else 1.6 * 1024 / LN2
    a_std = 0.8 * (800 if case["act"] == "gelu" else 1024 / LN2)
    gm, gs = _channels(rng, ffn, acc_std, gate_std)
    um, us = _channels(rng, ffn, acc_std, 4000)
    bias = _dev(np.rint(rng.normal(0, acc_std / 4, 2 * ffn)))
    return {"act": GELU if case["act"] == "gelu" else SILU, "gelu": gelu, "out_dy": _dyadic(32 / (a_std * 4000)), "mult": torch.cat([gm, um]),
            "shift": torch.cat([gs, us]), "bias": bias}


def _packed(gen, n, k, group, zeros):
    """4-bit weights, group scales and zero points as a program keeps them."""
    tiles, chunks = -(-n // 16), -(-k // 128)
    w = (torch.randn(tiles, chunks, 1024, 2, device="cuda", generator=gen) * 2.6).round_().clamp_(-8, 7).to(torch.int32) & 15
    shape = (tiles, chunks, 16, 128 // group)
    s = torch.randint(40, 256, shape, device="cuda", generator=gen).to(torch.uint8)
    z = torch.randint(-3, 4, shape, device="cuda", generator=gen).to(torch.int8) if zeros else None
    return {"w": (w[..., 0] | w[..., 1] << 4).to(torch.uint8), "scales": s, "zeros": z, "group": group, "n": n, "k": k}


def _acc_std(k, zeros):
    return 32 * math.sqrt(2.6 ** 2 + (4 if zeros else 0)) * 160 * math.sqrt(k)


def _prepare_products(case, gen, rng):
    t, k, kind = case["tokens"], case["hidden"], case["kind"]
    st = {"case": case, "a": _normal8(gen, 32, t, k)}
    if kind == "gated":
        st.update(_gate(case, rng, case["ffn"], 32 * 32 * math.sqrt(k)), w=_normal8(gen, 32, 2 * case["ffn"], k))
    elif kind == "w4_gated":
        st.update(_gate(case, rng, case["ffn"], _acc_std(k, case["zeros"])), gate=_packed(gen, case["ffn"], k, case["group"], case["zeros"]),
                  up=_packed(gen, case["ffn"], k, case["group"], case["zeros"]))
    else:
        n, std = case["n"], {"i8": 32, "i16": 3000, "i32": 300}[case["out"]]
        mult, shift = _channels(rng, n, _acc_std(k, case["zeros"]), std)
        st.update(weights=_packed(gen, n, k, case["group"], case["zeros"]), mult=mult, shift=shift, bias=_dev(np.rint(rng.normal(0, 5e4, n))),
                  res=_normal8(gen, 32, t, n) if case["out"] == "i16" else None, res_dy=_dyadic(90.0), clamp={"i8": 127, "i16": 32767, "i32": 2 ** 31 - 1}[case["out"]])
        st["out"] = torch.zeros(t, n, device="cuda", dtype={"i8": torch.int8, "i16": torch.int16, "i32": torch.int32}[case["out"]])
        return st
    st["out"] = torch.zeros(t, case["ffn"], device="cuda", dtype=torch.int8)
    return st


def _lengths(n, top):
    """n whole numbers from 0 to top, top first, in no order: the same for every seed."""
    return np.array([top] + [int((top + 1) * (0.6180339887498949 * i % 1.0)) for i in range(1, n)], np.int64)


def _prepare_logits(case, gen, rng):
    rows, vocab, masks = case["rows"], case["vocab"], case["masks"]
    lens, blens = _lengths(rows, case["tokens"]), _lengths(rows, case["biases"])
    start, bstart = np.concatenate([[0], np.cumsum(lens)]), np.concatenate([[0], np.cumsum(blens)])
    # words of a text: few of them often
    tokens = np.minimum(vocab - 1, (vocab * rng.random(start[-1]) ** 4)).astype(np.int64)
    step = LN2 / 64
    pen = rng.choice([1.0, 1.1, 1.3, 0.9], rows)
    return {"case": case, "x": (torch.randn(rows, vocab, device="cuda", generator=gen) * 300).round_().to(torch.int32),
            "params": _dev(np.array([[*_dyadic(1 / p), *_dyadic(p), round(f / step), round(g / step), m] for p, f, g, m in
                                     zip(pen, rng.choice([0, 0.4, 1.0], rows), rng.choice([0, 0.1, 0.5], rows),
                                         np.where(np.arange(rows) % 2 == 0, rng.integers(0, max(1, masks), rows), -1) if masks else np.full(rows, -1))])),
            "tokens": _dev(tokens), "token_start": _dev(start), "out_start": _dev(start[:-1] + (lens * rng.random(rows)).astype(np.int64)),
            "bias_ids": _dev(rng.integers(0, vocab, bstart[-1])), "bias_values": _dev(rng.integers(-500, 500, bstart[-1])), "bias_start": _dev(bstart),
            "masks": _dev(rng.integers(0, 2 ** 32, (masks, -(-vocab // 32))) & rng.integers(0, 2 ** 32, (masks, -(-vocab // 32))), torch.int64).to(torch.int32)
            if masks else None, "out": torch.zeros(rows, vocab, device="cuda", dtype=torch.int32)}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng([1321, 2101, seed])
    return (_prepare_logits if case["kind"] == "logits" else _prepare_products)(case, gen, rng)


# ---------------------------------------------------------------------------------------------- the plain forms
def _dy(x, m, s):
    """floor((x m + 2^(s-1)) / 2^s) of tensors of whole numbers, s >= 1."""
    return (x * m + (1 << (s - 1))) >> s


def _scaled(p):
    """The weights of a packed matrix with their zero points and group scales: whole numbers, [n, k]."""
    tiles, chunks, group = p["w"].shape[0], p["w"].shape[1], p["group"]
    w = p["w"].view(tiles, chunks, 4, 16, 2, 8)
    w = torch.stack([w & 15, w >> 4], 2).to(torch.int16)                                    # tile, chunk, half, q, row, half of half, byte
    w = ((w ^ 8) - 8).permute(0, 4, 1, 2, 5, 3, 6).reshape(16 * tiles, chunks * 128 // group, group)
    per_group = lambda x: x.permute(0, 2, 1, 3).reshape(16 * tiles, -1, 1).to(torch.int16)  # noqa: E731
    if p["zeros"] is not None:
        w = w - per_group(p["zeros"])
    return (w * per_group(p["scales"])).reshape(16 * tiles, -1)[:p["n"], :p["k"]]


def _sums(a, w, bias):
    """a w^T + bias, exact, inside 32 bits."""
    return (torch.matmul(a.double(), w.double().t()).long() + bias).clamp(LOW, 2 ** 31 - 1)


def _sigmoid(d):
    """The sigmoid of a distance d >= 0 in steps of ln2/64 with 15 bits, by i-exp."""
    z = d >> 6
    e = ((Q_B - (d & 63)) ** 2 + Q_C + ((1 << z) >> 1)) >> z
    e = torch.where(z < 16, e, 0)
    return (TOP * 2 ** 15 + (TOP + e) // 2) // (TOP + e)


def _gated(st, acc_g, acc_u):
    f, c = acc_g.shape[1], st["gelu"]
    m, s = st["mult"].long(), st["shift"].long()
    g, u = _dy(acc_g, m[:f], s[:f]), _dy(acc_u, m[f:], s[f:]).clamp(-32767, 32767)
    if st["act"] == GELU:
        g = g.clamp(-c["q_max"], c["q_max"])
        erf = torch.sign(g) * ((g.abs().clamp(max=-c["q_b"]) + c["q_b"]) ** 2 + c["q_c"])
        a = _dy(g * (erf + c["q_1"]), c["m"], c["s"]).clamp(-32767, 32767)
    else:
        g = g.clamp(-65535, 65535)
        p = _sigmoid(((g.abs() + 8) >> 4).clamp(max=1024))
        a = (g * torch.where(g < 0, 2 ** 15 - p, p) + 2 ** 14) >> 15
    st["out"].copy_(_dy(a * u, *st["out_dy"]).clamp(-127, 127))


def _plain_gated(st):
    f = st["case"]["ffn"]
    acc = _sums(st["a"], st["w"], st["bias"])
    _gated(st, acc[:, :f], acc[:, f:])


def _plain_w4_gated(st):
    f = st["case"]["ffn"]
    _gated(st, _sums(st["a"], _scaled(st["gate"]), st["bias"][:f]), _sums(st["a"], _scaled(st["up"]), st["bias"][f:]))


def _plain_w4(st):
    v = _dy(_sums(st["a"], _scaled(st["weights"]), st["bias"]), st["mult"].long(), st["shift"].long())
    if st["res"] is not None:
        v = v + _dy(st["res"].long(), *st["res_dy"])
    st["out"].copy_(v.clamp(-st["clamp"], st["clamp"]))


def _plain_logits(st):
    rows, vocab = st["x"].shape
    p = st["params"].long()
    n = torch.arange(st["tokens"].numel(), device="cuda")
    row = torch.searchsorted(st["token_start"][1:].long(), n, right=True)
    made = n >= st["out_start"].long()[row]
    count = torch.zeros(2, rows, vocab, dtype=torch.int64, device="cuda")
    count.index_put_((made.long(), row, st["tokens"].long()), torch.ones_like(n), accumulate=True)
    bias = torch.zeros(rows, vocab, dtype=torch.int64, device="cuda")
    brow = torch.searchsorted(st["bias_start"][1:].long(), torch.arange(st["bias_ids"].numel(), device="cuda"), right=True)
    bias.index_put_((brow, st["bias_ids"].long()), st["bias_values"].long(), accumulate=True)
    x = st["x"].long()
    up, down = _dy(x, p[:, 0:1], p[:, 1:2]), _dy(x, p[:, 2:3], p[:, 3:4])
    v = torch.where(count.sum(0) > 0, torch.where(x > 0, up, down).clamp(LOW, 2 ** 31 - 1), x)
    v = (v - p[:, 4:5] * (count[1] > 0) - p[:, 5:6] * count[1] + bias).clamp(LOW + 1, 2 ** 31 - 1)
    v = torch.where(x == LOW, LOW, v)
    if st["masks"] is not None:
        t = torch.arange(vocab, device="cuda")
        open_ = (st["masks"][:, t // 32] >> (t % 32)) & 1
        v = torch.where((p[:, 6:7] < 0) | (open_[p[:, 6].clamp(min=0)] == 1), v, LOW)
    st["out"].copy_(v)


# ---------------------------------------------------------------------------------------------- a pass
def _own_gate(B, st, ldw):
    if "desc" not in st:          # what a program makes once
        c = st["gelu"]
        gate = B.GateParams(st["act"], B.GeluParams(c["q_b"], c["q_c"], c["q_1"], c["q_max"], B.Dyadic(c["m"], c["s"])), B.Dyadic(*st["out_dy"]))
        st["desc"] = B.GatedDesc(st["case"]["tokens"], st["case"]["ffn"], st["case"]["hidden"], st["a"].shape[1], ldw, st["out"].shape[1], gate)
    return st["desc"]


def _own_weights(B, st, name):
    key = "own_" + name
    if key not in st:
        p = st[name]
        st[key] = B.W4Weights(p["w"].data_ptr(), p["scales"].data_ptr(), p["zeros"].data_ptr() if p["zeros"] is not None else None, p["group"])
    return st[key]


def _own_gated(B, st):
    B.ibert_gemm_i8_gated(_own_gate(B, st, st["w"].shape[1]), st["a"], st["w"], st["bias"], st["mult"], st["shift"], st["out"])


def _own_w4_gated(B, st):
    B.ibert_gemm_w4_gated(_own_gate(B, st, 0), st["a"], _own_weights(B, st, "gate"), _own_weights(B, st, "up"), st["bias"], st["mult"], st["shift"], st["out"])


def _own_w4(B, st):
    if "desc" not in st:
        n, k = st["case"]["n"], st["case"]["hidden"]
        st["desc"] = B.W4Desc(st["case"]["tokens"], n, k, {"i8": B.I8, "i16": B.I16, "i32": B.I32}[st["case"]["out"]], k, n, n, st["clamp"], B.Dyadic(*st["res_dy"]))
    B.ibert_gemm_w4_requant(st["desc"], st["a"], _own_weights(B, st, "weights"), st["bias"], st["mult"], st["shift"], st["res"], st["out"])


def _own_logits(B, st):
    if "desc" not in st:
        c = st["case"]
        st["desc"] = B.LogitsDesc(c["rows"], c["vocab"], c["vocab"], c["vocab"], st["tokens"].numel(), st["bias_ids"].numel(), c["masks"],
                                  st["masks"].shape[1] if c["masks"] else 0)
    B.ibert_logits_adjust_i(st["desc"], st["x"], st["params"], st["tokens"], st["token_start"], st["out_start"], st["bias_ids"], st["bias_values"],
                            st["bias_start"], st["masks"], st["out"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2101_01321_amd import binding as B
        {"gated": _own_gated, "w4": _own_w4, "w4_gated": _own_w4_gated, "logits": _own_logits}[kind](B, state)
    else:
        {"gated": _plain_gated, "w4": _plain_w4, "w4_gated": _plain_w4_gated, "logits": _plain_logits}[kind](state)
    return {"out": state["out"]}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _rounded(x, m, s):
    """x m / 2^s to the nearest whole number, halves up: the quotient and what it leaves."""
    q = torch.div(x * m, 2 ** s if isinstance(s, int) else torch.ones_like(s) << s, rounding_mode="floor")
    left = x * m - q * (2 ** s if isinstance(s, int) else torch.ones_like(s) << s)
    return q + (2 * left >= (2 ** s if isinstance(s, int) else torch.ones_like(s) << s))


def _whole_weight(p, n):
    """Rows n of a packed matrix, each weight found by its offset."""
    k, chunks, group = torch.arange(p["k"], device="cuda"), p["w"].shape[1], p["group"]
    n = n[:, None]
    byte = p["w"].reshape(-1)[(n // 16 * chunks + k // 128) * 1024 + k % 32 // 8 * 256 + n % 16 * 16 + k % 64 // 32 * 8 + k % 8].long()
    w = torch.where(k % 128 < 64, byte % 16, byte // 16)
    w = torch.where(w > 7, w - 16, w)
    at = ((n // 16 * chunks + k // 128) * 16 + n % 16) * (128 // group) + k % 128 // group
    if p["zeros"] is not None:
        w = w - p["zeros"].reshape(-1)[at].long()
    return (w * p["scales"].reshape(-1)[at].long()).double()


def _exact_products(st):
    """Channels by the hundred, tokens by the thousand; SiLU from a list of its sigmoids."""
    case, a, out = st["case"], st["a"], torch.empty_like(st["out"])
    half = [TOP * 2.0 ** 15 / (TOP + (math.floor(((Q_B - d % 64) ** 2 + Q_C) / 2 ** (d // 64) + 0.5) if d < 1024 else 0)) for d in range(1025)]
    half = torch.tensor([math.floor(h + 0.5) for h in half], device="cuda")
    m, s, bias, c = st["mult"].long(), st["shift"].long(), st["bias"].long(), st["gelu"] if "gelu" in st else None
    for n0 in range(0, out.shape[1], 1024):
        n = torch.arange(n0, min(n0 + 1024, out.shape[1]), device="cuda")
        parts = {"gated": lambda: [st["w"][n].double(), st["w"][n + out.shape[1]].double()], "w4": lambda: [_whole_weight(st["weights"], n)],
                 "w4_gated": lambda: [_whole_weight(st["gate"], n), _whole_weight(st["up"], n)]}[case["kind"]]()
        for t0 in range(0, out.shape[0], 2048):
            t = slice(t0, t0 + 2048)
            v = []
            for i, w in enumerate(parts):
                ch = n + i * out.shape[1]
                acc = ((w @ a[t].double().t()).t().round().long() + bias[ch]).clamp(-2 ** 31, 2 ** 31 - 1)
                v.append(_rounded(acc, m[ch], s[ch]))
            if case["kind"] == "w4":
                y = v[0] + (_rounded(st["res"][t, n0:n0 + 1024].long(), *st["res_dy"]) if st["res"] is not None else 0)
                out[t, n0:n0 + 1024] = y.clamp(-st["clamp"], st["clamp"]).to(out.dtype)
                continue
            g, u = v[0], v[1].clamp(-32767, 32767)
            if case["act"] == "gelu":
                g = g.clamp(-c["q_max"], c["q_max"])
                poly = (torch.minimum(g.abs(), torch.full_like(g, -c["q_b"])) + c["q_b"]).square() + c["q_c"]
                act = _rounded(torch.where(g < 0, g * (c["q_1"] - poly), torch.where(g > 0, g * (c["q_1"] + poly), 0)), c["m"], c["s"]).clamp(-32767, 32767)
            else:
                g = g.clamp(-65535, 65535)
                sg = half[torch.div(g.abs() + 8, 16, rounding_mode="floor").clamp(max=1024)]
                act = _rounded(g, torch.where(g < 0, 32768 - sg, sg), 15)
            out[t, n0:n0 + 1024] = _rounded(act * u, *st["out_dy"]).clamp(-127, 127).to(torch.int8)
    return {"out": out}


def _exact_logits(st):
    """A row at a time on the host."""
    x, p, out = st["x"].cpu().numpy(), st["params"].cpu().tolist(), np.empty(st["x"].shape, np.int64)
    tokens, ids, values = (st[k].cpu().numpy() for k in ("tokens", "bias_ids", "bias_values"))
    start, made, bstart = (st[k].cpu().tolist() for k in ("token_start", "out_start", "bias_start"))
    masks = st["masks"].cpu().numpy().view(np.uint32) if st["masks"] is not None else None
    for r, (um, us, dm, ds, presence, frequency, mask) in enumerate(p):
        v = x[r].astype(np.int64)
        seen, n = np.unique(tokens[start[r]:start[r + 1]]), np.bincount(tokens[made[r]:start[r + 1]], minlength=v.size)
        v[seen] = [(int(a) * m + 2 ** (s - 1)) // 2 ** s for a in v[seen] for m, s in [(um, us) if a > 0 else (dm, ds)]]
        v = np.clip(v, -2 ** 31, 2 ** 31 - 1) - presence * (n > 0) - frequency * n
        np.add.at(v, ids[bstart[r]:bstart[r + 1]], values[bstart[r]:bstart[r + 1]])
        v = np.clip(v, -2 ** 31 + 1, 2 ** 31 - 1)
        v[x[r] == -2 ** 31] = -2 ** 31
        if mask >= 0:
            bits = np.unpackbits(masks[mask].view(np.uint8), bitorder="little")[:v.size]
            v[bits == 0] = -2 ** 31
        out[r] = v
    return {"out": torch.from_numpy(out).to("cuda", torch.int32)}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_logits(st) if case["kind"] == "logits" else _exact_products(st)


# ---------------------------------------------------------------------------------------------- what a pass takes
def work(case):
    if case["kind"] == "logits":
        cells, tokens, biases = case["rows"] * case["vocab"], int(_lengths(case["rows"], case["tokens"]).sum()), int(_lengths(case["rows"], case["biases"]).sum())
        return {"bytes": 8 * cells + 4 * tokens + 8 * biases + min(case["masks"], (case["rows"] + 1) // 2) * -(-case["vocab"] // 32) * 4 + 40 * case["rows"], "flops": 0}
    t, k, kind = case["tokens"], case["hidden"], case["kind"]
    n = case["n"] if kind == "w4" else 2 * case["ffn"]
    weight = n * k if kind == "gated" else n * k // 2 + n * -(-k // case["group"]) * (2 if case["zeros"] else 1)
    out = t * case["n"] * {"i8": 1, "i16": 3, "i32": 4}[case["out"]] if kind == "w4" else t * case["ffn"]
    return {"bytes": t * k + weight + 12 * n + out, "flops": 2 * t * n * k}
