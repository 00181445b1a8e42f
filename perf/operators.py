"""The decoder-side operators on cases that can be timed: page tables of an INT8 key/value cache, the rotation of queries and
keys with the append to that cache, and attention over it, for single new tokens and for prompts.

Everything is integer and exact.  With `own` false the operators run in their plain form, elementary torch operations; with
`own` true they are the library's entry points.  Both read and write the same buffers.

The cache of a layer holds pages of P tokens (P = 64 * 2^k); within a page and head, 64 tokens at a time:
  K[page][head][t / 16][d / 16][t % 16][d % 16]
  V[page][head][t / 64][d / 16][t % 16 / 4][d % 16][t % 64 / 16][t % 4]
"""
import math

import numpy as np
import torch

own = False

Q_B, Q_C = 124, 8180          # i-exp's constants floor(b/S), floor(c/(a S^2)) at S = ln2/64
ONE = 1 << 14                 # cos and sin of the rotation table


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one request gets one more token: what a page costs when nothing is large; pure latency
        {"name": "pages_b1", "kind": "pages", "batch": 1, "page": 64, "max_len": 2048, "mix": "decode"},
        # a step of a full server: most requests decode, some come with a prompt, some have ended and return their pages
        {"name": "pages_b512_mixed", "kind": "pages", "batch": 512, "page": 64, "max_len": 8192, "mix": "mixed"},
        # one decode step of a small batch, heads as the Base shape has them
        {"name": "rotary_b5_h12_d64", "kind": "rotary", "heads_q": 12, "heads_kv": 12, "dim": 64, "rot": 64, "layout": "half", "norm": False,
         "batch": 5, "tokens": 5, "page": 64, "scaling": "none"},
        # packed prompts of uneven lengths, a quarter of each head rotated, neighbours paired, positions scaled linearly
        {"name": "rotary_t2741_part", "kind": "rotary", "heads_q": 16, "heads_kv": 16, "dim": 64, "rot": 16, "layout": "interleaved", "norm": False,
         "batch": 11, "tokens": 2741, "page": 128, "scaling": "linear"},
        # a large prefill step with grouped heads, normalised queries and keys, positions of a stretched context
        {"name": "rotary_t16384_norm", "kind": "rotary", "heads_q": 32, "heads_kv": 8, "dim": 128, "rot": 128, "layout": "half", "norm": True,
         "batch": 4, "tokens": 16384, "page": 64, "scaling": "ramp"},
        # the first answer token of one short question, heads as the Base shape has them; latency
        {"name": "decode_b1_l77_h12", "kind": "attention", "heads_q": 12, "heads_kv": 12, "dim": 64, "batch": 1, "q_len": 1, "kv_len": 77,
         "window": 0, "sinks": 0, "page": 64},
        # a serving batch in full swing: grouped heads, requests of every age
        {"name": "decode_b64_l4096_h32", "kind": "attention", "heads_q": 32, "heads_kv": 8, "dim": 128, "batch": 64, "q_len": 1, "kv_len": 4096,
         "window": 0, "sinks": 0, "page": 64},
        # one request with a whole book in its context
        {"name": "decode_b1_l131071", "kind": "attention", "heads_q": 32, "heads_kv": 8, "dim": 128, "batch": 1, "q_len": 1, "kv_len": 131071,
         "window": 0, "sinks": 0, "page": 128},
        # long chats with a sliding window and a few first tokens that stay visible, heads as the Large shape has them
        {"name": "decode_b32_window", "kind": "attention", "heads_q": 16, "heads_kv": 16, "dim": 64, "batch": 32, "q_len": 1, "kv_len": 16384,
         "window": 1021, "sinks": 4, "page": 64},
        # a batch of uneven prompts
        {"name": "prompt_b8_q489_h16", "kind": "attention", "heads_q": 16, "heads_kv": 16, "dim": 64, "batch": 8, "q_len": 489, "kv_len": 489,
         "window": 0, "sinks": 0, "page": 64},
        # one long prompt, grouped heads
        {"name": "prompt_b1_q4096_h32", "kind": "attention", "heads_q": 32, "heads_kv": 8, "dim": 128, "batch": 1, "q_len": 4096, "kv_len": 4096,
         "window": 0, "sinks": 0, "page": 64},
        # the next piece of two long prompts behind what the cache already holds, with window and sinks
        {"name": "piece_b2_q1500_window", "kind": "attention", "heads_q": 32, "heads_kv": 8, "dim": 128, "batch": 2, "q_len": 1500, "kv_len": 9001,
         "window": 2048, "sinks": 16, "page": 256},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["pages", "rotary", "decode", "prompt"], [2, 3, 5, 4])[0]
    page = rng.choice([64, 128, 256])
    if kind == "pages":
        return {"kind": kind, "batch": _log_int(rng, 1, 512), "page": page, "max_len": _log_int(rng, 128, 8192), "mix": rng.choice(["decode", "mixed"])}
    dim = rng.choice([64, 128])
    heads_kv = rng.choice([1, 2, 4, 8, 12])
    heads_q = heads_kv * rng.choice([1, 2, 3, 4, 7, 8]) if heads_kv <= 4 else heads_kv * rng.choice([1, 2, 4])
    heads_q = min(heads_q, 32 // heads_kv * heads_kv) if heads_kv < 12 else 12
    if kind == "rotary":
        tokens = _log_int(rng, 1, 16384)
        return {"kind": kind, "heads_q": heads_q, "heads_kv": heads_kv, "dim": dim, "rot": rng.choice([dim, dim, dim // 2, dim // 4]),
                "layout": rng.choice(["half", "interleaved"]), "norm": rng.random() < 0.5, "batch": _log_int(rng, 1, min(tokens, 256)), "tokens": tokens,
                "page": page, "scaling": rng.choice(["none", "linear", "base", "ramp"])}
    window = rng.choice([0, 0, _log_int(rng, 64, 4096)])
    sinks = rng.choice([0, 4, rng.randint(1, 100)]) if window else 0
    case = {"kind": "attention", "heads_q": heads_q, "heads_kv": heads_kv, "dim": dim, "window": window, "sinks": sinks, "page": page}
    if kind == "decode":
        batch = _log_int(rng, 1, 256)
        return dict(case, batch=batch, q_len=1, kv_len=_log_int(rng, 1, 262144 // batch if batch > 2 else 131071))
    q_len = _log_int(rng, 2, 4096)
    batch = _log_int(rng, 1, max(1, 4096 // q_len))
    return dict(case, batch=batch, q_len=q_len, kv_len=min(4096, q_len + rng.choice([0, _log_int(rng, 1, 4096)])))


# ---------------------------------------------------------------------------------------------- inputs
def _spread(n, lo, hi):
    """n whole numbers from lo to hi, hi first, in no order: the lengths of a case, the same for every seed."""
    return np.array([hi] + [lo + int((hi - lo + 1) * (0.6180339887498949 * i % 1.0)) for i in range(1, n)], np.int64)


def _dyadic(real):
    """(m, s) with real ~ m / 2^s and m of 31 bits."""
    f, e = math.frexp(real)
    m = round(f * 2 ** 31)
    return (m >> 1, 30 - e) if m == 1 << 31 else (m, 31 - e)


def _normal8(gen, std, *shape):
    return (torch.randn(shape, device="cuda", generator=gen) * std).round_().clamp_(-127, 127).to(torch.int8)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda", dtype)


def _pages_of(lens, page):
    return -(-lens // page)


def _block_table(rng, lens, page):
    """Pages of sequences that have `lens` tokens, scattered over the cache, and the number of pages in it."""
    need = _pages_of(lens, page)
    width, total = max(1, int(need.max())), int(need.sum()) + 3
    pool, table, at = rng.permutation(total), np.zeros((len(lens), width), np.int64), 0
    for i, n in enumerate(need):
        table[i, :n] = pool[at:at + n]
        at += n
    return table, total


def _attention_lens(case):
    if case["q_len"] == 1:
        return np.ones(case["batch"], np.int64), _spread(case["batch"], max(1, case["kv_len"] // 4), case["kv_len"])
    q = _spread(case["batch"], max(1, case["q_len"] // 2), case["q_len"])
    return q, q + case["kv_len"] - case["q_len"]


def _prepare_attention(case, gen, rng):
    q_lens, kv_lens = _attention_lens(case)
    hq, hk, d, page = case["heads_q"], case["heads_kv"], case["dim"], case["page"]
    table, total = _block_table(rng, kv_lens, page)
    rows, cells = int(q_lens.sum()), total * hk * page * d
    s_qk, s_v = 6.0 / 127, 4.0 / 127
    return {"case": case, "rows": rows, "num_pages": total, "max_pages": table.shape[1], "max_q": int(q_lens.max()), "max_kv": int(kv_lens.max()),
            "q": _normal8(gen, 127 / 4, rows, hq * d), "k": _normal8(gen, 127 / 4, cells), "v": _normal8(gen, 127 / 4, cells),
            "table": _dev(table), "q_start": _dev(np.concatenate([[0], np.cumsum(q_lens)])), "kv_len": _dev(kv_lens),
            "scores_dy": _dyadic(s_qk * s_qk / math.sqrt(d) * 64 / math.log(2)), "out_dy": _dyadic(s_v / (s_v / 3) / 65536),
            "out": torch.zeros(rows, hq * d, dtype=torch.int8, device="cuda")}


def _freqs(case):
    """Radians a position for each pair, the context stretched by 4 in one of the usual ways."""
    rot, base, factor, first = case["rot"], 10000.0, 4.0, 4096
    if case["scaling"] == "base":
        base *= factor ** (rot / (rot - 2))
    theta = base ** (-np.arange(0, rot, 2) / rot)
    if case["scaling"] == "linear":
        theta = theta / factor
    if case["scaling"] == "ramp":       # turns over the first context: over 32 as they are, under 1 stretched, between them a mix
        keep = np.clip((first * theta / (2 * math.pi) - 1) / 31, 0, 1)
        theta = theta * (keep + (1 - keep) / factor)
    return theta


def _prepare_rotary(case, gen, rng):
    hq, hk, d, page, batch, tokens = (case[k] for k in ("heads_q", "heads_kv", "dim", "page", "batch", "tokens"))
    runs = np.full(batch, tokens // batch) + (np.arange(batch) < tokens % batch)
    start = _spread(batch, 0, 8191)
    # the pages that this step writes to; those of the earlier tokens play no part in it
    first = start % page
    table, total = _block_table(rng, first + runs, page)
    positions = np.concatenate([s + np.arange(n) for s, n in zip(start, runs)])
    slots = np.concatenate([t[(f + np.arange(n)) // page] * page + (f + np.arange(n)) % page for t, f, n in zip(table, first, runs)])
    max_pos = 8192 + int(runs.max())
    angle = np.arange(max_pos)[:, None] * _freqs(case)
    rope = np.stack([np.rint(np.cos(angle) * ONE), np.rint(np.sin(angle) * ONE)], -1)
    gamma = lambda: _dev(np.rint(rng.normal(1.0, 0.1, d) * 8192))  # noqa: E731
    # x / rms has 10 fractional bits, times gamma at 13, >> 11: 12 are left; then 14 of the rotation, and 4 standard deviations to 127
    dy = _dyadic(127 / 4 / 4096 / ONE) if case["norm"] else _dyadic(0.9 / ONE)
    return {"case": case, "rows": tokens, "num_pages": total, "max_pos": max_pos, "qkv": _normal8(gen, 127 / 4, tokens, (hq + 2 * hk) * d),
            "rope": _dev(rope, torch.int16), "positions": _dev(positions), "slots": _dev(slots), "q_dy": dy, "k_dy": dy, "v_dy": _dyadic(0.8),
            "q_gamma": gamma() if case["norm"] else None, "k_gamma": gamma() if case["norm"] else None, "gamma_shift": 11,
            "q": torch.zeros(tokens, hq * d, dtype=torch.int8, device="cuda"),
            "k": torch.zeros(total * hk * page * d, dtype=torch.int8, device="cuda"), "v": torch.zeros(total * hk * page * d, dtype=torch.int8, device="cuda")}


def _pages_lens(case):
    """Lengths before and after a step."""
    batch, top = case["batch"], case["max_len"]
    before = _spread(batch, 1, top - 1)
    after = before + 1
    if case["mix"] == "mixed":
        k = np.arange(batch) % 16
        before, after = np.where(k == 5, 0, before), np.where(k == 5, np.minimum(before, 512), np.where(k == 11, 0, after))
    return before, after


def _prepare_pages(case, gen, rng):
    batch, page = case["batch"], case["page"]
    before, after = _pages_lens(case)
    order = rng.permutation(batch)
    before, after = before[order], after[order]
    had, wants = _pages_of(before, page), _pages_of(after, page)
    width = -(-case["max_len"] // page)
    # every page is some sequence's or waits in the ring
    held, spare = int(had.sum()), int(np.maximum(0, wants - had).sum()) + 5
    num = held + spare
    ids = rng.permutation(num)
    table = np.zeros((batch, width), np.int64)
    table[np.arange(width) < had[:, None]] = ids[:held]
    head = int(rng.integers(0, num))
    ring = np.zeros(num, np.int64)
    ring[(head + np.arange(spare)) % num] = ids[held:]
    rows = int(np.maximum(0, after - before).sum()) + batch % 7
    new = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"case": case, "rows": rows, "num_pages": num, "max_pages": width, "before": _dev(before), "after": _dev(after), "table": _dev(table),
            "ring": _dev(ring), "ring_in": _dev(np.array([head, spare])), "ring_out": new(3), "q_start": new(batch + 1), "kv_len": new(batch),
            "slots": new(rows), "positions": new(rows)}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng([2101, 1321, seed])
    return {"pages": _prepare_pages, "rotary": _prepare_rotary, "attention": _prepare_attention}[case["kind"]](case, gen, rng)


# ---------------------------------------------------------------------------------------------- the plain forms
def _dy(x, dy):
    """floor((x m + 2^(s-1)) / 2^s) of a tensor of whole numbers."""
    m, s = dy
    return (x.to(torch.int64) * m + (1 << s >> 1)) >> s


def _to8(x):
    return x.clamp(-127, 127).to(torch.int8)


def _plain_pages(st):
    page, R, rows, table = st["case"]["page"], st["num_pages"], st["rows"], st["table"]
    width = table.shape[1]
    before, after = st["before"].long().clamp(min=0), st["after"].long().clamp(min=0)
    head, count = st["ring_in"][0].long(), st["ring_in"][1].long()
    had, wants = (before + page - 1) // page, (after + page - 1) // page
    need, new = (wants - had).clamp(min=0), (after - before).clamp(min=0)
    fits = (wants <= width) & ((need == 0) | (need.cumsum(0) <= count)) & ((new == 0) | (new.cumsum(0) <= rows))
    after = torch.where(fits, after, before)
    wants = torch.where(fits, wants, had)
    need, back, new = (wants - had).clamp(min=0), (had - wants).clamp(min=0), (after - before).clamp(min=0)
    p = torch.arange(width, device=table.device)
    at = p + (need.cumsum(0) - need - had)[:, None]
    taken = (p >= had[:, None]) & (p < wants[:, None])
    to = p + (back.cumsum(0) - back - wants)[:, None]
    gone = (p >= wants[:, None]) & (p < had[:, None])
    ring = torch.cat([st["ring"], st["ring"][:1]])                       # (one more, for what is not returned)
    ring.index_put_((torch.where(gone, (head + count + to) % R, R).reshape(-1),), table.reshape(-1))
    table.copy_(torch.where(taken, st["ring"][(head + at) % R], table))
    st["ring"].copy_(ring[:R])
    st["ring_out"].copy_(torch.stack([(head + need.sum()) % R, count - need.sum() + back.sum(), (~fits).sum()]))
    st["q_start"][1:] = new.cumsum(0)
    st["kv_len"].copy_(after)
    t = torch.arange(rows, device=table.device)
    ends = new.cumsum(0)
    seq = torch.searchsorted(ends, t, right=True).clamp(max=len(ends) - 1)
    real = t < ends[-1]
    pos = torch.where(real, before[seq] + t - (ends - new)[seq], 0)
    st["positions"].copy_(pos)
    st["slots"].copy_(torch.where(real, table[seq, pos // page].long() * page + pos % page, -1))


def _plain_rotary(st):
    c = st["case"]
    hq, hk, d, rot, page = c["heads_q"], c["heads_kv"], c["dim"], c["rot"], c["page"]
    x = st["qkv"].view(-1, hq + 2 * hk, d).int()
    cos, sin = st["rope"][st["positions"].long()].long().unbind(-1)

    def turned(u, gamma, dy):
        if gamma is not None:
            var = ((u * u).sum(-1, keepdim=True).long() << 16) // d
            sigma = var.double().sqrt().floor().long().clamp(min=1)
            n = (u * ((1 << 30) // sigma)) >> 12
            u = ((n * gamma + (1 << st["gamma_shift"] >> 1)) >> st["gamma_shift"]).clamp(-32767, 32767)
        u = u.long()
        r, rest = u[..., :rot], u[..., rot:] * ONE
        a, b = (r[..., :rot // 2], r[..., rot // 2:]) if c["layout"] == "half" else (r[..., 0::2], r[..., 1::2])
        cs, sn = cos[:, None], sin[:, None]
        a, b = a * cs - b * sn, a * sn + b * cs
        r = torch.cat([a, b], -1) if c["layout"] == "half" else torch.stack([a, b], -1).flatten(-2)
        return _to8(_dy(torch.cat([r, rest], -1), dy))

    st["q"].copy_(turned(x[:, :hq], st["q_gamma"], st["q_dy"]).flatten(1))
    k, v = turned(x[:, hq:hq + hk], st["k_gamma"], st["k_dy"]), _to8(_dy(x[:, hq + hk:], st["v_dy"]))
    pg, t = st["slots"].long() // page, st["slots"].long() % page
    kc, vc = st["k"].view(-1, hk, page // 16, d // 16, 16, 16), st["v"].view(-1, hk, page // 64, d // 16, 4, 16, 4, 4)
    kc[pg, :, t // 16, :, t % 16] = k.view(-1, hk, d // 16, 16)
    vc[pg, :, t // 64, :, t % 16 // 4, :, t % 64 // 16, t % 4] = v.view(-1, hk, d // 16, 16)


def _plain_attention(st):
    c = st["case"]
    hq, hk, d, page, window = c["heads_q"], c["heads_kv"], c["dim"], c["page"], c["window"]
    batch, n, group = c["batch"], st["max_q"], hq // hk
    start, kv = st["q_start"].long(), st["kv_len"].long()
    i = torch.arange(n, device=kv.device)
    real = i < (start[1:] - start[:-1])[:, None]
    at = (start[:-1, None] + i).clamp(max=st["rows"] - 1)
    q = st["q"].view(-1, hk, group, d)[at].float().permute(0, 2, 1, 3, 4).reshape(batch, hk, n * group, d)
    pages = st["table"].long()
    k = st["k"].view(-1, hk, page // 16, d // 16, 16, 16)[pages].float().permute(0, 2, 1, 3, 5, 4, 6).reshape(batch, hk, -1, d)
    v = st["v"].view(-1, hk, page // 64, d // 16, 4, 16, 4, 4)[pages].double().permute(0, 2, 1, 3, 7, 5, 8, 4, 6).reshape(batch, hk, -1, d)
    scores = torch.matmul(q, k.transpose(2, 3)).view(batch, hk, n, group, -1)              # exact: under 2^24
    j = torch.arange(k.shape[2], device=kv.device)
    pos = (kv - (start[1:] - start[:-1]))[:, None] + i                                      # of each query
    seen = j <= pos[..., None]
    if window:
        seen &= (j > pos[..., None] - window) | (j < c["sinks"])
    seen = (seen & real[..., None])[:, None, :, None]
    top = scores.masked_fill(~seen, -math.inf).amax(-1, keepdim=True).clamp(min=-2.0 ** 23)
    far = _dy((top - scores).clamp(min=0), st["scores_dy"])
    z = far >> 6
    w = ((Q_B - (far & 63)) ** 2 + Q_C + ((1 << z.clamp(max=20)) >> 1)) >> z.clamp(max=20)
    w = torch.where(seen & (z < 16), w, 0).double()
    total = w.sum(-1, keepdim=True).long()
    mean = torch.matmul(w.view(batch, hk, n * group, -1), v).view(batch, hk, n, group, d).long()
    mean = (mean * ((1 << 48) // total.clamp(min=1))) >> 32
    o = _to8(_dy(mean, st["out_dy"])).permute(0, 2, 1, 3, 4).reshape(batch, n, hq * d)
    rows = torch.empty(st["rows"] + 1, hq * d, dtype=torch.int8, device=o.device)           # (one more, for what lies past a sequence's end)
    rows[torch.where(real, at, st["rows"])] = o
    st["out"].copy_(rows[:-1])


# ---------------------------------------------------------------------------------------------- a pass
def _own_cache(B, st):
    c = st["case"]
    return B.KvCache(st["k"].data_ptr(), st["v"].data_ptr(), c["heads_kv"], c["dim"], c["page"], st["num_pages"])


def _own_pages(B, st):
    B.ibert_page_tables_i(st["before"], st["after"], st["case"]["batch"], st["case"]["page"], st["num_pages"], st["ring_in"], st["ring"], st["ring_out"],
                          st["table"], st["max_pages"], st["rows"], st["q_start"], st["kv_len"], st["slots"], st["positions"])


def _own_rotary(B, st):
    c = st["case"]
    if "desc" not in st:          # what a program makes once
        st["desc"] = B.RotaryDesc(c["heads_q"], c["rot"], B.ROTARY_HALF if c["layout"] == "half" else B.ROTARY_INTERLEAVED, st["max_pos"],
                                  B.Dyadic(*st["q_dy"]), B.Dyadic(*st["k_dy"]), B.Dyadic(*st["v_dy"]), st["gamma_shift"], st["gamma_shift"])
        st["cache"] = _own_cache(B, st)
    B.ibert_rotary_append_i(st["desc"], st["cache"], st["qkv"], st["qkv"].shape[1], st["rope"], st["positions"], st["slots"], st["q_gamma"], st["k_gamma"],
                            st["rows"], st["q"], st["q"].shape[1])


def _own_attention(B, st):
    c = st["case"]
    if "desc" not in st:
        st["desc"] = B.PagedAttentionDesc(c["heads_q"], c["window"], c["sinks"], B.Dyadic(*st["scores_dy"]), B.Dyadic(*st["out_dy"]))
        st["cache"] = _own_cache(B, st)
        size = B.ibert_paged_attention_workspace_bytes(st["desc"], st["cache"], c["batch"], st["rows"], st["max_q"], st["max_kv"])
        st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.ibert_paged_attention_i(st["desc"], st["cache"], st["q"], st["q"].shape[1], st["table"], st["max_pages"], st["q_start"], st["kv_len"], c["batch"],
                              st["rows"], st["max_q"], st["max_kv"], st["out"], st["out"].shape[1], st["ws"])


_OUT = {"pages": ("table", "ring", "ring_out", "q_start", "kv_len", "slots", "positions"), "rotary": ("q", "k", "v"), "attention": ("out",)}


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2101_01321_amd import binding as B
        {"pages": _own_pages, "rotary": _own_rotary, "attention": _own_attention}[kind](B, state)
    else:
        {"pages": _plain_pages, "rotary": _plain_rotary, "attention": _plain_attention}[kind](state)
    return {name: state[name] for name in _OUT[kind]}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _exact_pages(st):
    c, page, R = st["case"], st["case"]["page"], st["num_pages"]
    before, after, table, ring = (st[k].cpu().numpy().astype(np.int64) for k in ("before", "after", "table", "ring"))
    head, count = (int(x) for x in st["ring_in"].cpu())
    slots, positions, q_start, kv, ends = [], [], [0], [], []
    asked_pages = asked_rows = taken = refused = 0
    old = ring.copy()
    for b in range(len(before)):
        had, wants, new = -(-before[b] // page), -(-after[b] // page), max(0, after[b] - before[b])
        asked_pages += max(0, wants - had)
        asked_rows += new
        ok = wants <= table.shape[1] and (wants <= had or asked_pages <= count) and (new == 0 or asked_rows <= st["rows"])
        refused += not ok
        kv.append(after[b] if ok else before[b])
        if ok:
            for p in range(had, wants):
                table[b, p] = old[(head + taken) % R]
                taken += 1
            ends += [table[b, p] for p in range(wants, had)]
            for p in range(before[b], after[b]):
                positions.append(p)
                slots.append(table[b, p // page] * page + p % page)
        q_start.append(len(slots))
    for k, p in enumerate(ends):
        ring[(head + count + k) % R] = p
    pad = st["rows"] - len(slots)
    return {"table": table, "ring": ring, "ring_out": np.array([(head + taken) % R, count - taken + len(ends), refused]), "q_start": np.array(q_start),
            "kv_len": np.array(kv), "slots": np.array(slots + [-1] * pad), "positions": np.array(positions + [0] * pad)}


def _exact_rotary(st):
    c = st["case"]
    hq, hk, d, rot, page = c["heads_q"], c["heads_kv"], c["dim"], c["rot"], c["page"]
    x = st["qkv"].cpu().numpy().astype(np.int64).reshape(-1, hq + 2 * hk, d)
    cs = st["rope"].cpu().numpy().astype(np.int64)[st["positions"].cpu().numpy()][:, None]
    slots = st["slots"].cpu().numpy().astype(np.int64)

    def rounded(y, dy):
        return np.clip((y * dy[0] + (1 << (dy[1] - 1))) >> dy[1], -127, 127)

    def one(y, gamma, dy):
        if gamma is not None:
            n = np.square(y).sum(-1) * 65536 // d
            root = np.sqrt(n.astype(np.float64)).astype(np.int64)
            root = np.maximum(1, root + ((root + 1) ** 2 <= n) - (root ** 2 > n))
            y = ((y * ((1 << 30) // root)[..., None]) >> 12) * gamma.cpu().numpy().astype(np.int64)
            y = np.clip((y + (1 << (st["gamma_shift"] - 1))) >> st["gamma_shift"], -32767, 32767)
        i = np.arange(rot // 2)
        first, second = (i, i + rot // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        z = y * ONE
        z[..., first] = y[..., first] * cs[..., 0] - y[..., second] * cs[..., 1]
        z[..., second] = y[..., first] * cs[..., 1] + y[..., second] * cs[..., 0]
        return rounded(z, dy)
    k, v = np.zeros(st["k"].numel(), np.int8), np.zeros(st["v"].numel(), np.int8)
    head, dim = np.arange(hk)[:, None], np.arange(d)
    base = (slots // page)[:, None, None] * (hk * page * d) + head * (page * d)
    t = (slots % page)[:, None, None]
    k[base + t // 16 * (16 * d) + dim // 16 * 256 + t % 16 * 16 + dim % 16] = one(x[:, hq:hq + hk], st["k_gamma"], st["k_dy"])
    v[base + t // 64 * (64 * d) + dim // 16 * 1024 + t % 16 // 4 * 256 + dim % 16 * 16 + t % 64 // 16 * 4 + t % 4] = rounded(x[:, hq + hk:], st["v_dy"])
    return {"q": one(x[:, :hq], st["q_gamma"], st["q_dy"]).reshape(-1, hq * d).astype(np.int8), "k": k, "v": v}


def _exact_attention(st):
    """A sequence and a key head at a time, cells found by their offsets, weights from a list."""
    c = st["case"]
    hq, hk, d, page = c["heads_q"], c["heads_kv"], c["dim"], c["page"]
    weight = [((Q_B - f % 64) ** 2 + Q_C) / 2 ** (f // 64) for f in range(1024)]
    weight = torch.tensor([math.floor(w + 0.5) for w in weight] + [0], dtype=torch.float64, device="cuda")
    start, lens, dim = st["q_start"].tolist(), st["kv_len"].tolist(), torch.arange(d, device="cuda")
    out = torch.zeros_like(st["out"])
    for b, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        page_of, t = st["table"][b].long()[t // page], t % page
        pos = torch.arange(start[b], start[b + 1], device="cuda") - start[b + 1] + n
        far = pos[:, None] - torch.arange(n, device="cuda")
        seen = far >= 0
        if c["window"]:
            seen &= (far < c["window"]) | (torch.arange(n, device="cuda") < c["sinks"])
        for h in range(hk):
            base = ((page_of * hk + h) * (page * d))[:, None]
            k = st["k"][base + (t // 16 * 16 * d + t % 16 * 16)[:, None] + dim // 16 * 256 + dim % 16].double()
            v = st["v"][base + (t // 64 * 64 * d + t % 16 // 4 * 256 + t % 64 // 16 * 4 + t % 4)[:, None] + dim // 16 * 1024 + dim % 16 * 16].double()
            for g in range(h * (hq // hk), (h + 1) * (hq // hk)):
                s = st["q"][start[b]:start[b + 1], g * d:(g + 1) * d].double() @ k.T
                s = torch.where(seen, s, -torch.inf)
                m, sh = st["scores_dy"]
                off = torch.where(seen, (s.amax(1, keepdim=True) - s).nan_to_num(0, 0, 0), 0).long()
                w = torch.where(seen, weight[((off * m + (1 << (sh - 1))) >> sh).clamp(max=1024)], 0.0)
                total = w.sum(1, keepdim=True).long()
                r = torch.where(total > 0, 2 ** 48 // total.clamp(min=1), 0)
                r = ((w @ v).long() * r) >> 32
                m, sh = st["out_dy"]
                out[start[b]:start[b + 1], g * d:(g + 1) * d] = ((r * m + (1 << (sh - 1))) >> sh).clamp(-127, 127).to(torch.int8)
    return {"out": out}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(st)
    got = (_exact_pages if case["kind"] == "pages" else _exact_rotary)(st)
    return {name: torch.from_numpy(np.ascontiguousarray(a)).to(st[name].dtype).reshape(st[name].shape) for name, a in got.items()}


# ---------------------------------------------------------------------------------------------- what a pass takes
def _visible(case):
    """Over all queries, the positions that each sees; and the positions that any query of a sequence sees."""
    pairs = cells = 0
    window, sinks = case["window"], case["sinks"]
    for n, kv in zip(*(x.tolist() for x in _attention_lens(case))):
        pos = np.arange(kv - n, kv)
        if not window:
            pairs, cells = pairs + int((pos + 1).sum()), cells + kv
            continue
        low = np.maximum(0, pos - window + 1)
        pairs += int((pos + 1 - low + np.minimum(sinks, low)).sum())
        cells += int(kv - low[0] + min(sinks, low[0]))
    return pairs, cells


def work(case):
    if case["kind"] == "pages":
        before, after = _pages_lens(case)
        moved = np.abs(_pages_of(after, case["page"]) - _pages_of(before, case["page"])).sum()
        rows = np.maximum(0, after - before).sum()
        return {"bytes": int(16 * case["batch"] + 8 * moved + 8 * rows + 24), "flops": 0}
    hq, hk, d = case["heads_q"], case["heads_kv"], case["dim"]
    if case["kind"] == "rotary":
        cells = case["tokens"] * (hq + 2 * hk) * d
        return {"bytes": 2 * cells + case["tokens"] * (2 * case["rot"] + 8), "flops": 6 * cells}
    pairs, cells = _visible(case)
    rows = int(_attention_lens(case)[0].sum())
    return {"bytes": 2 * cells * hk * d + 2 * rows * hq * d + 4 * case["batch"] * 2, "flops": 4 * pairs * hq * d}
