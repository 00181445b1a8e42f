"""The decoder attention on the GPU against the oracle, bit for bit: page tables, rotation with append, attention over the paged
cache, and the three together as a decoder would run them."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import oracle
import decoder_util as U


def libs():
    import torch
    import gpu_util as G
    from paper_2101_01321_amd import binding as B
    return torch, G, B


def same(got, want, what):
    got = got.cpu().numpy() if hasattr(got, "cpu") else got
    bad = np.flatnonzero(got.reshape(-1) != want.reshape(-1))
    assert bad.size == 0, "%s: %d of %d differ, first at %d: %s, not %s" % (what, bad.size, want.size, bad[0], got.reshape(-1)[bad[0]], want.reshape(-1)[bad[0]])


# ------------------------------------------------------------------------------------------- page tables
class DevicePages:
    def __init__(self, p):
        torch, G, B = libs()
        self.p = p
        self.t = {k: G.to_dev(getattr(p, k)) for k in ("before", "after", "ring_in", "ring", "table")}
        guard = lambda n: torch.full((n + 8,), 77, dtype=torch.int32, device=G.DEV)      # noqa: E731
        self.o = {"ring_out": guard(3), "q_start": guard(len(p.before) + 1), "kv_len": guard(len(p.before)), "slots": guard(p.rows), "positions": guard(p.rows)}
        self.n = {"ring_out": 3, "q_start": len(p.before) + 1, "kv_len": len(p.before), "slots": p.rows, "positions": p.rows}

    def call(self, stream=None):
        _, _, B = libs()
        p, t, o = self.p, self.t, self.o
        B.ibert_page_tables_i(t["before"], t["after"], len(p.before), p.page, p.num, t["ring_in"], t["ring"], o["ring_out"], t["table"], p.width, p.rows, o["q_start"],
                              o["kv_len"], o["slots"], o["positions"], stream)

    def check(self):
        want = self.p.oracle()
        same(self.t["table"], want["table"], "table")
        same(self.t["ring"], want["ring"], "ring")
        for k, n in self.n.items():
            same(self.o[k][:n], want[k], k)
            assert bool((self.o[k][n:] == 77).all()), "wrote past the end of " + k
        return want


def _pages_cases():
    rng = np.random.default_rng(11)
    yield "one token", U.Pages(0, [0], [1], 64)
    yield "one more", U.Pages(1, [64], [65], 64)
    yield "no page needed", U.Pages(2, [65], [66], 64)
    yield "nothing to do", U.Pages(3, [65, 0], [65, 0], 64, extra_rows=4)
    yield "no sequences", U.Pages(4, [], [], 64, rows=9)
    yield "no rows", U.Pages(5, [100, 70], [50, 0], 64, rows=0)
    yield "negative lengths", U.Pages(6, [-5, 70, -2 ** 31], [3, -1, 0], 64)
    for batch in (2, 63, 64, 65, 512, 513, 1500, 8192):
        yield "mixed %d" % batch, U.Pages(batch, *U.mixed_lengths(rng, batch, 700 if batch < 2000 else 130), 64, extra_rows=batch % 5)
    yield "wide pages", U.Pages(7, *U.mixed_lengths(rng, 40, 5000), 1024)
    yield "too few pages", U.Pages(8, *U.mixed_lengths(rng, 600, 700), 64, count=400)
    yield "no pages at all", U.Pages(9, [10, 64, 0], [11, 65, 1], 64, count=0, more_pages=0)
    yield "too few rows", U.Pages(10, *U.mixed_lengths(rng, 600, 300), 128, rows=3000)
    yield "a row of the table too short", U.Pages(11, [60, 5, 128], [300, 6, 129], 64, width=2)
    yield "asked for far too much", U.Pages(12, [0, 5, 10, 0], [2 ** 31 - 1, 2 ** 31 - 1, 11, 2 ** 31 - 1], 64, width=4, count=5, rows=64)


@pytest.mark.parametrize("name,case", list(_pages_cases()), ids=lambda v: v.replace(" ", "_") if isinstance(v, str) else "")
def test_page_tables(gpu, name, case):
    torch, G, B = libs()
    G.say("page tables: " + name)
    d = DevicePages(case)
    d.call()
    torch.cuda.synchronize()
    want = d.check()
    if name.startswith(("too", "no pages", "a row", "asked")):
        assert want["ring_out"][2] > 0


def _pages_of_many_rounds():
    rng = np.random.default_rng(14)
    yield "150000 rows of wide pages", U.Pages(20, [0, 5, 1024, 0, 100], [30000, 30005, 31024, 30000, 30100], 1024, extra_rows=300)
    yield "8.8 million rows, 137500 pages", U.Pages(21, [0] * 20 + [7000], [440000] * 20 + [0], 64, extra_rows=7)
    yield "no rows, 38998 pages back", U.Pages(22, rng.integers(129 * 64, 130 * 64, 300), np.zeros(300), 64, rows=0)
    yield "one row, pages back from every other sequence", U.Pages(23, [9000, 64] * 400 + [64], [100, 64] * 400 + [65], 64)
    yield "three rows for many, pages back", U.Pages(24, [5000, 63] * 700, [0, 65] * 700, 64, rows=3)


@pytest.mark.parametrize("name,case", list(_pages_of_many_rounds()), ids=lambda v: v.replace(" ", "_") if isinstance(v, str) else "")
def test_page_tables_of_more_than_one_round(gpu, name, case):
    # more rows than 256 workgroups have threads, and more pages than a launch that is sized by few rows has
    torch, G, B = libs()
    G.say("page tables: " + name)
    d = DevicePages(case)
    for _ in range(2):
        d.call()
        torch.cuda.synchronize()
        want = d.check()
        if _ == 0:                           # once more from what was there before
            for k in ("ring", "table"):
                d.t[k].copy_(torch.from_numpy(getattr(case, k)))
    assert (want["ring_out"][2] > 0) == name.startswith("three")


def test_page_tables_of_the_most_rows_there_can_be(gpu):
    # 2^31 - 1 rows, and asked for one more: who asked first is refused for want of pages, who asks next, without a page, for want of rows; who asks for none is not
    torch, G, B = libs()
    most, i32 = 2 ** 31 - 1, lambda a: torch.tensor(a, dtype=torch.int32, device=G.DEV)     # noqa: E731
    before, after, ring_in, ring = i32([0, 1, 70, 5]), i32([most, 2, 3, 5]), i32([1, 4]), i32([0, 4, 5, 6, 7, 0, 0, 0])
    table = i32([[0, 0], [0, 0], [1, 2], [3, 0]])
    ring_out, q_start, kv_len = i32([77] * 3), i32([77] * 5), i32([77] * 4)
    slots, positions = (torch.full((most,), 77, dtype=torch.int32, device=G.DEV) for _ in range(2))
    G.say("page tables: %d rows" % most)
    B.ibert_page_tables_i(before, after, 4, 64, 8, ring_in, ring, ring_out, table, 2, most, q_start, kv_len, slots, positions)
    torch.cuda.synchronize()
    assert ring_out.tolist() == [1, 5, 2] and q_start.tolist() == [0] * 5 and kv_len.tolist() == [0, 1, 3, 5]
    assert ring.tolist() == [0, 4, 5, 6, 7, 2, 0, 0] and table.tolist() == [[0, 0], [0, 0], [1, 2], [3, 0]]
    for t, want in ((slots, -1), (positions, 0)):
        for part in t.split(1 << 28):
            assert bool((part == want).all())


def test_page_tables_clamp_what_the_ring_says(gpu):
    # a head and a count outside the ring are taken as the nearest inside; nothing else is touched
    torch, G, B = libs()
    for head, count in ((-3, 5), (10 ** 9, 3), (2, -1), (1, 10 ** 9)):
        case = U.Pages(13, [10, 64, 0], [11, 65, 1], 64)
        case.ring_in = np.array([head, count], np.int32)
        G.say("page tables: ring says %d, %d" % (head, count))
        d = DevicePages(case)
        d.call()
        torch.cuda.synchronize()
        case.ring_in = np.array([np.clip(head, 0, case.num - 1), np.clip(count, 0, case.num)], np.int32)
        d.check()


# ------------------------------------------------------------------------------------------- rotation and append
def run_rotary(case, stream=None):
    torch, G, B = libs()
    tk, tv, tq = G.to_dev(case.k0), G.to_dev(case.v0), G.to_dev(case.q0)
    desc, cache = case.descs(tk, tv)
    dev = lambda a: None if a is None else G.to_dev(a)      # noqa: E731
    B.ibert_rotary_append_i(desc, cache, G.to_dev(case.qkv), case.qkv.shape[1], dev(case.cs if case.R else None), dev(case.positions), dev(case.slots), dev(case.gq), dev(case.gk),
                            case.rows, tq, case.q0.shape[1], stream)
    torch.cuda.synchronize()
    return tq, tk, tv


ROTARY = [  # rows, hq, hk, D, R, interleaved, page, q_norm, k_norm, ld, skip
    (1, 1, 1, 64, 64, False, 64, False, False, 0, ()), (1, 1, 1, 128, 128, True, 64, True, True, 0, ()),
    (7, 12, 12, 64, 64, False, 64, False, False, 0, (2, 3)), (130, 12, 12, 64, 32, True, 128, False, False, 48, (0, 7, 129)),
    (65, 32, 8, 128, 128, False, 64, True, True, 16, (64,)), (33, 7, 1, 128, 48, True, 256, True, False, 0, ()),
    (64, 5, 5, 64, 16, False, 64, False, True, 32, (1,)), (200, 2, 2, 128, 16, False, 512, False, False, 0, ()),
    (31, 3, 3, 64, 0, False, 64, True, False, 0, ()), (300, 4, 2, 128, 112, False, 64, True, True, 0, range(100, 140)), (1, 64, 8, 128, 64, True, 64, False, False, 0, ())]


@pytest.mark.parametrize("args", ROTARY, ids=lambda a: "t%d_q%d_k%d_d%d_r%d_%s_n%d%d" % (a[0], a[1], a[2], a[3], a[4], "il" if a[5] else "half", a[7], a[8]))
def test_rotary_append(gpu, args):
    torch, G, B = libs()
    rows, hq, hk, D, R, inter, page, qn, kn, ld, skip = args
    case = U.Rotary(rows + R, rows, hq, hk, D, R, inter, page, qn, kn, ld, skip)
    G.say("rotary %s" % (args,))
    for got, want, what in zip(run_rotary(case), case.oracle(), "qkv"):
        same(got, want, what)


@pytest.mark.parametrize("dy", [(0, 0), (1, 0), (-(2 ** 31 - 1), 62), (2 ** 31 - 1, 31), (2 ** 30, 32), (2 ** 31 - 1, 33), (12345, 7)])
def test_rotary_append_of_any_dyadic(gpu, dy):
    torch, G, B = libs()
    case = U.Rotary(3, 10, 3, 1, 64, 32, False, 64, False, True)
    case.q_dy = case.k_dy = case.v_dy = dy
    G.say("rotary dyadic %s" % (dy,))
    for got, want, what in zip(run_rotary(case), case.oracle(), "qkv"):
        same(got, want, what)


@pytest.mark.parametrize("D,page", [(64, 64), (128, 256)])
def test_values_of_rows_that_fill_blocks(gpu, D, page):
    # runs of rows on runs of slots that start and end anywhere, with gaps, rows without a slot and runs that meet in one block
    torch, G, B = libs()
    runs = [(0, 64), (70, 64), (200, 300), (640, 1), (641, 63), (704, 128), (900, 59), (960, 63), (1024, 64), (1090, 190), (1281, 3), (1290, 4), (1299, 5), (1310, 2), (1312, 1), (1344, 130)]
    rows = sum(n for _, n in runs) + 5
    case = U.Rotary(D, rows, 2, 2, D, 32, False, page)
    order = np.random.default_rng(D).permutation(len(runs))
    slots = np.concatenate([np.arange(s, s + n) for s, n in (runs[i] for i in order)] + [np.full(5, -1)])
    case.slots = slots.astype(np.int32)
    for skip in ((), (3, 64, 300), range(0, rows, 65)):
        for i in skip:
            case.slots[i] = -1
        G.say("values in blocks, D %d, %d rows without a slot" % (D, len(skip)))
        for got, want, what in zip(run_rotary(case), case.oracle(), "qkv"):
            same(got, want, what)


@pytest.mark.parametrize("dy", [(0, 0), (1, 0), (-1, 0), (3, 1), (127, 8), (2 ** 31 - 1, 0), (-(2 ** 31 - 1), 8), (2 ** 30, 9), (2 ** 30, 30), (2 ** 31 - 1, 32), (-(2 ** 30), 33), (2 ** 31 - 1, 40), (5, 62)])
def test_values_of_any_dyadic(gpu, dy):
    torch, G, B = libs()
    case = U.Rotary(9, 200, 1, 1, 64, 0, False, 64)
    case.slots = (np.arange(200) + 10).astype(np.int32)
    case.qkv[:, 128:192] = np.arange(200 * 64).reshape(200, 64) % 256 - 128          # every value there is
    case.v_dy = dy
    G.say("values, dyadic %s" % (dy,))
    for got, want, what in zip(run_rotary(case), case.oracle(), "qkv"):
        same(got, want, what)


def test_rotary_append_of_many_rows(gpu):
    torch, G, B = libs()
    for D, rows in ((64, 3001), (128, 1403)):
        case = U.Rotary(D, rows, 8, 2, D, D, D == 64, 64, D == 128, D == 128)
        # prompts stand in a row: the slots of a sequence follow each other
        case.slots = (np.arange(rows) + 17).astype(np.int32)
        G.say("rotary %d rows of D %d" % (rows, D))
        for got, want, what in zip(run_rotary(case), case.oracle(), "qkv"):
            same(got, want, what)


TEAMS = ROTARY + [  # the same, of heads of 128 whose pieces are whole: odd numbers of heads, one norm, none or a part rotated, rows that leave the last workgroup partly filled
    (67, 7, 1, 128, 128, False, 64, True, False, 16, (0, 5, 66)), (129, 9, 3, 128, 64, True, 128, False, True, 0, ()), (257, 5, 5, 128, 32, False, 64, True, True, 32, range(0, 257, 9)),
    (63, 3, 3, 128, 0, False, 64, False, False, 0, ()), (95, 15, 5, 128, 96, True, 256, True, True, 0, (94,)), (1, 1, 1, 128, 96, False, 64, True, True, 0, ()),
    (2, 2, 2, 128, 128, True, 64, False, False, 0, (1,)), (65, 33, 11, 128, 128, True, 64, True, False, 0, ()), (40, 64, 2, 128, 64, False, 64, False, True, 48, ())]


@pytest.mark.parametrize("args", TEAMS, ids=lambda a: "t%d_q%d_k%d_d%d_r%d_%s_n%d%d" % (a[0], a[1], a[2], a[3], a[4], "il" if a[5] else "half", a[7], a[8]))
def test_rotary_append_of_one_and_two_heads_a_team(gpu, args):
    torch, G, B = libs()
    rows, hq, hk, D, R, inter, page, qn, kn, ld, skip = args
    case = U.Rotary(rows + R + 1, rows, hq, hk, D, R, inter, page, qn, kn, ld, skip)
    # heads whose roots are far apart beside each other: nothing, one unit, the most there is
    case.qkv[0, D:2 * D] = 0
    case.qkv[0, 2 * D - 1] = 1
    case.qkv[rows // 2, :D] = -128
    want = case.oracle()
    for heads in (1, 2):
        G.say("rotary %s, %d heads a team" % (args, heads))
        B.ibert_rotary_override(heads)
        try:
            got = run_rotary(case)
        finally:
            B.ibert_rotary_override(-1)
        assert B.lib().ibert_last_kernel().decode().endswith(", %d>" % (heads if D == 128 and R % 32 == 0 else 1))
        for g, w, what in zip(got, want, "qkv"):
            same(g, w, "%s, %d heads a team" % (what, heads))


@pytest.mark.parametrize("rows,hq,hk,R,inter,qn,kn,heads", [
    (8192, 32, 8, 128, False, True, True, 2), (8191, 32, 8, 128, True, True, True, 1), (37450, 7, 1, 64, True, True, False, 2), (29128, 9, 3, 32, False, False, True, 2),
    (20165, 13, 1, 0, False, False, False, 2), (2033, 129, 1, 96, False, True, True, 2), (16384, 16, 4, 112, False, False, True, 1)])
def test_rotary_append_by_its_rule_for_many_rows(gpu, rows, hq, hk, R, inter, qn, kn, heads):
    # on both sides of 262144 heads of queries; half of the rows in runs as a prompt has them, the others anywhere, some without a slot
    torch, G, B = libs()
    case = U.Rotary(rows + hq, rows, hq, hk, 128, R, inter, 64, qn, kn, 16, range(5, rows, 997))
    free = np.setdiff1d(np.arange(case.pages * 64, dtype=np.int32), case.slots[rows // 2:])
    run = case.slots[:rows // 2] >= 0
    case.slots[:rows // 2][run] = free[:int(run.sum())]
    G.say("rotary by rule: %d rows, %d + %d heads, R %d" % (rows, hq, hk, R))
    got = run_rotary(case)
    assert B.lib().ibert_last_kernel().decode().endswith(", %d>" % heads)
    for g, w, what in zip(got, case.oracle(), "qkv"):
        same(g, w, what)


# ------------------------------------------------------------------------------------------- attention
class DeviceAttention:
    def __init__(self, case, max_q=None, max_kv=None, plain_rows=False):
        torch, G, B = libs()
        self.case = case
        self.tq, self.tk, self.tv, self.table, self.kv = (G.to_dev(a) for a in (case.q, case.k, case.v, case.table, case.kv_len))
        self.start = None if plain_rows else G.to_dev(case.q_start)
        self.out = torch.cat([G.to_dev(case.out).reshape(-1), torch.full((64,), 77, dtype=torch.int8, device=G.DEV)])
        self.desc, self.cache = case.descs(self.tk, self.tv)
        self.max_q = max(1, int(case.n.max(initial=1))) if max_q is None else max_q
        self.max_kv = int(case.kv.max(initial=0)) if max_kv is None else max_kv
        size = B.ibert_paged_attention_workspace_bytes(self.desc, self.cache, case.batch, case.rows, self.max_q, self.max_kv)
        self.ws = torch.randint(-128, 128, (size + 256,), dtype=torch.int8, device=G.DEV) if size else None
        self.size = size

    def call(self, stream=None):
        _, _, B = libs()
        c = self.case
        B.ibert_paged_attention_i(self.desc, self.cache, self.tq, c.q.shape[1], self.table, c.table.shape[1], self.start, self.kv, c.batch, c.rows, self.max_q, self.max_kv,
                                  self.out, c.out.shape[1], None if self.ws is None else self.ws[:self.size], stream)

    def result(self):
        torch, _, _ = libs()
        torch.cuda.synchronize()
        assert bool((self.out[-64:] == 77).all()), "wrote past the end"
        return self.out[:-64].reshape(self.case.out.shape)


def check_attention(case, **kw):
    """The call as it is, and in each of its four forms."""
    torch, G, B = libs()
    want = case.oracle()
    for form in (B.PAGED_TWICE, B.PAGED_ONE, B.PAGED_SPLIT, B.PAGED_PROMPT, -1):
        G.say("attention form %d q%d k%d d%d page %d n %s kv %s window %d sinks %d" % (form, case.hq, case.hk, case.D, case.page, case.n[:8].tolist(), case.kv[:8].tolist(), case.window,
                                                                                       case.sinks))
        B.ibert_paged_attention_override(form)
        try:
            d = DeviceAttention(case, **kw)
            d.call()
            same(d.result(), want, "out, form %d" % form)
        finally:
            B.ibert_paged_attention_override(-1)
    return d, want


@pytest.mark.parametrize("n,kv,hq,hk,D,window,kernel", [
    ([1], [77], 12, 12, 64, 0, "paged_row_kernel"), ([1] * 64, [3000] * 64, 8, 2, 128, 0, "paged_row_kernel"), ([1], [3000], 8, 2, 128, 0, "paged_join_kernel"),
    ([1], [9000], 8, 2, 128, 500, "paged_row_kernel"), ([8], [5000], 8, 2, 128, 0, "paged_join_kernel"), ([64], [200], 8, 2, 128, 0, "paged_attention_kernel"),
    ([200] * 3, [200] * 3, 8, 2, 128, 0, "paged_attention_kernel"), ([200] * 14, [200] * 14, 8, 2, 128, 0, "paged_prompt_kernel")])
def test_attention_takes_the_kernel_that_the_rule_names(gpu, n, kv, hq, hk, D, window, kernel):
    torch, G, B = libs()
    case = U.Attention(60, hq, hk, D, 64, n, kv, window)
    G.say("attention by rule: %s" % kernel)
    d = DeviceAttention(case)
    d.call()
    d.result()
    assert B.lib().ibert_last_kernel().decode().startswith(kernel)


@pytest.mark.parametrize("hq,hk,D,page", [(1, 1, 64, 64), (12, 12, 64, 64), (8, 2, 128, 64), (7, 1, 128, 128), (16, 1, 64, 256), (40, 2, 64, 64), (17, 1, 128, 64)])
def test_attention_of_single_rows(gpu, hq, hk, D, page):
    kv = [1, 2, 63, 64, 65, 127, 128, 129, 0, 300, 700]
    check_attention(U.Attention(hq + D, hq, hk, D, page, [1] * len(kv), kv))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (64, 0), (63, 4), (200, 64), (100, 65), (65, 1000), (5000, 4), (128, 130)])
def test_attention_window_and_sinks(gpu, window, sinks):
    kv = [1, 64, 65, 200, 201, 333, 512, 1000]
    check_attention(U.Attention(window + sinks, 4, 2, 64, 64, [1] * len(kv), kv, window, sinks))
    check_attention(U.Attention(window + sinks, 3, 1, 128, 128, [50, 1, 70, 200], [50, 90, 400, 333], window, sinks))


@pytest.mark.parametrize("hq,hk,D,page", [(1, 1, 64, 64), (12, 12, 64, 64), (8, 2, 128, 64), (7, 1, 128, 256), (32, 2, 64, 128), (5, 1, 64, 64)])
def test_attention_of_prompts(gpu, hq, hk, D, page):
    check_attention(U.Attention(hq, hq, hk, D, page, [1, 2, 0, 65, 130, 16], [1, 2, 30, 65, 140, 300]))


def test_attention_of_a_long_prompt(gpu):
    check_attention(U.Attention(21, 4, 1, 128, 64, [517], [517]))
    check_attention(U.Attention(22, 2, 2, 64, 64, [1030, 3], [1111, 1000]))


def test_attention_of_a_long_context(gpu):
    # one and a few rows on long caches: the work of a row is split and joined
    check_attention(U.Attention(23, 4, 1, 64, 64, [1], [70001], std=20.0))
    check_attention(U.Attention(24, 2, 2, 128, 256, [1, 1, 1], [20000, 0, 9]))
    check_attention(U.Attention(25, 4, 2, 64, 64, [3, 1, 2], [9000, 5, 4097], 0, 0))
    check_attention(U.Attention(26, 2, 1, 64, 64, [1, 1], [40000, 30000], 20000, 100))


def test_attention_at_the_longest_context(gpu):
    # 131072 keys that all weigh the same, values at the ends of their range: the largest sums there are
    case = U.Attention(27, 1, 1, 64, 1024, [1], [131072])
    case.q[:] = 0
    case.v[:] = np.where(np.arange(case.v.size) % 64 < 32, 127, -127)
    d, want = check_attention(case)
    assert np.all(np.abs(want[0, :64]) >= 126)
    # one key 380 steps above all others, whose weight there is 256 h - 128: the low halves are all at the end of their range
    assert oracle.weight(380) % 256 == 128
    case.s_dy = (1 << 30, 30)                    # a raw score is a step
    case.k[:] = 0
    case.q[0, 0] = 4
    t = 5
    case.k[int(case.table[0, 0]) * 1024 * 64 + t * 16] = 95
    check_attention(case)


def test_attention_rows_that_see_nothing(gpu):
    # more rows than the cache has tokens: the first ones come before every key
    d, want = check_attention(U.Attention(28, 6, 3, 64, 64, [5, 40, 1, 3], [2, 30, 0, 0]))
    assert np.all(want[:3, :6 * 64] == 0) and want[3].any()


def test_attention_of_padded_batches_and_strides(gpu):
    # rows behind the last sequence, columns behind those of a row: left as they were
    for n, kv in (([1, 1, 1], [100, 5, 64]), ([30, 1, 9], [100, 5, 64])):
        case = U.Attention(29, 4, 2, 64, 64, n, kv, pad=11, ld=32)
        d, want = check_attention(case, max_q=50, max_kv=5000)
        same(want[int(sum(n)):], case.out[int(sum(n)):], "padding")


def test_attention_of_one_row_a_sequence_needs_no_starts(gpu):
    check_attention(U.Attention(30, 8, 2, 128, 64, [1] * 5, [1, 700, 64, 0, 129], pad=2), plain_rows=True)


def test_attention_without_keys(gpu):
    for n in ([1, 1], [70, 3]):
        d, want = check_attention(U.Attention(46, 4, 2, 64, 64, n, [0, 0], pad=2))
        assert not want[:int(sum(n))].any()


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (131071, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_attention_of_the_largest_windows(gpu, window, sinks):
    # (rows before the first key among them)
    check_attention(U.Attention(47, 4, 2, 64, 64, [1, 1, 1], [100, 300, 0], window, sinks))
    check_attention(U.Attention(48, 4, 2, 64, 64, [100, 70, 5], [50, 200, 2], window, sinks))


def test_offsets_beyond_32_bits(gpu):
    # a cache of over 4 GB for each of K and V, whose last pages are the ones in use
    torch, G, B = libs()
    D, hk, page = 128, 8, 256
    high = (4 << 30) // (page * hk * D) + 50
    case = U.Attention(49, 16, hk, D, page, [1, 40], [600, 700])
    rot = U.Rotary(50, 70, 16, hk, D, D, False, page)
    cells = (high + max(case.pages, rot.pages)) * page * hk * D
    tk, tv = (torch.zeros(cells, dtype=torch.int8, device=G.DEV) for _ in range(2))
    base = high * page * hk * D
    assert base > 1 << 32
    tk[base:base + case.k.size], tv[base:base + case.v.size] = G.to_dev(case.k), G.to_dev(case.v)
    want = case.oracle()
    for form in (B.PAGED_TWICE, B.PAGED_ONE, B.PAGED_SPLIT, B.PAGED_PROMPT):
        G.say("attention in a cache of %d MB, form %d" % (cells >> 20, form))
        B.ibert_paged_attention_override(form)
        try:
            d = DeviceAttention(case)
            d.table += high
            d.cache = B.KvCache(tk.data_ptr(), tv.data_ptr(), hk, D, page, high + case.pages)
            d.call()
            same(d.result(), want, "out, form %d" % form)
        finally:
            B.ibert_paged_attention_override(-1)
    want = rot.oracle()
    tk[base:base + rot.k0.size], tv[base:base + rot.v0.size] = G.to_dev(rot.k0), G.to_dev(rot.v0)
    tq = G.to_dev(rot.q0)
    desc, cache = rot.descs(tk, tv)
    cache.num_pages = high + rot.pages
    G.say("rotary into a cache of %d MB" % (cells >> 20))
    B.ibert_rotary_append_i(desc, cache, G.to_dev(rot.qkv), rot.qkv.shape[1], G.to_dev(rot.cs), G.to_dev(rot.positions), G.to_dev(rot.slots + high * page), None, None, rot.rows, tq,
                            rot.q0.shape[1])
    torch.cuda.synchronize()
    same(tq, want[0], "q")
    same(tk[base:base + rot.k0.size], want[1], "k")
    same(tv[base:base + rot.v0.size], want[2], "v")


def test_attention_of_rows_that_start_anywhere_allowed(gpu):
    # q 16 bytes into its buffer, out 4 bytes into its own
    torch, G, B = libs()
    for n, kv in (([1, 1], [90, 3000]), ([70, 5], [90, 200])):
        case = U.Attention(51, 4, 2, 64, 64, n, kv, ld=16)
        want = case.oracle()
        for form in (B.PAGED_TWICE, B.PAGED_ONE, B.PAGED_SPLIT, B.PAGED_PROMPT):
            G.say("attention of shifted rows, form %d" % form)
            B.ibert_paged_attention_override(form)
            try:
                d = DeviceAttention(case)
                tq, to = torch.zeros(case.q.size + 16, dtype=torch.int8, device=G.DEV), torch.full((case.out.size + 4,), 77, dtype=torch.int8, device=G.DEV)
                tq[16:], to[4:] = G.to_dev(case.q).reshape(-1), G.to_dev(case.out).reshape(-1)
                d.tq, d.out = tq[16:], to[4:]
                d.call()
                torch.cuda.synchronize()
                same(to[4:], want.reshape(-1), "out, form %d" % form)
                assert bool((to[:4] == 77).all())
            finally:
                B.ibert_paged_attention_override(-1)


def test_attention_leaves_rows_beyond_max_q_len(gpu):
    torch, G, B = libs()
    case = U.Attention(31, 3, 1, 64, 64, [40, 10, 21], [60, 10, 90])
    for most in (1, 7, 20, 30):
        G.say("attention: at most %d rows of each sequence" % most)
        d = DeviceAttention(case, max_q=most)
        d.call()
        want, seen = case.oracle(), np.concatenate([np.arange(k) < most for k in case.n])
        same(d.result(), np.where(seen[:, None], want, case.out), "out")


def _rows_beyond_the_bound():
    rng = np.random.default_rng(81)
    yield "few", U.Attention(82, 3, 1, 64, 64, [40, 10, 21, 1, 0], [60, 10, 90, 70, 5], pad=3), (1, 7, 20, 30)
    yield "few, width 128, a window", U.Attention(83, 8, 2, 128, 64, [5, 130, 64, 17], [200, 400, 64, 30], 50, 5), (3, 5, 16, 65, 129)
    n = np.zeros(200, np.int64)
    n[rng.permutation(200)[:20]] = rng.integers(100, 200, 20)
    yield "tiles that are counted", U.Attention(84, 8, 2, 64, 64, n, n + rng.integers(0, 90, 200), pad=4), (131,)
    n = np.where(rng.random(200) < 0.5, 1, 0)
    n[[7, 150]], n[60:64] = 500, 90
    yield "tiles that are counted, single rows apart", U.Attention(85, 8, 2, 64, 64, n, n + rng.integers(0, 300, 200), pad=4), (301, 77)
    yield "single rows apart", U.Attention(86, 8, 2, 128, 64, [1] * 20 + [600] + [1] * 10, [700] * 20 + [650] + [300] * 10), (333,)


@pytest.mark.parametrize("name,case,bounds", list(_rows_beyond_the_bound()), ids=lambda v: v.replace(" ", "_") if isinstance(v, str) else "")
def test_attention_of_every_form_leaves_rows_beyond_max_q_len(gpu, name, case, bounds):
    torch, G, B = libs()
    want = case.oracle()
    for most in bounds:
        seen = np.zeros(case.rows, bool)
        seen[:int(case.n.sum())] = np.concatenate([np.arange(k) < most for k in case.n])
        for form in (B.PAGED_TWICE, B.PAGED_ONE, B.PAGED_SPLIT, B.PAGED_PROMPT, -1):
            G.say("attention, %s: at most %d rows of each sequence, form %d" % (name, most, form))
            B.ibert_paged_attention_override(form)
            try:
                d = DeviceAttention(case, max_q=most)
                d.call()
                same(d.result(), np.where(seen[:, None], want, case.out), "out, form %d, at most %d" % (form, most))
            finally:
                B.ibert_paged_attention_override(-1)
        if not name.startswith("few"):
            assert B.lib().ibert_last_kernel().decode().startswith("paged_prompt_kernel")


def test_attention_clamps_lengths_and_pages(gpu):
    torch, G, B = libs()
    case = U.Attention(32, 4, 2, 64, 64, [1, 1, 1], [100, 128, 70])
    d = DeviceAttention(case, max_kv=100)
    d.kv.copy_(torch.tensor([100, 10 ** 9, -7], dtype=torch.int32))
    G.say("attention: lengths beyond their bounds")
    d.call()
    case.kv_len[:] = (100, 100, 0)
    same(d.result(), case.oracle(), "lengths")
    case = U.Attention(33, 4, 2, 64, 64, [1, 2], [100, 128])
    d = DeviceAttention(case)
    wild = case.table.copy()
    wild[0, 0], wild[1, 1] = -1, 2 ** 31 - 1
    d.table.copy_(torch.from_numpy(wild))
    G.say("attention: pages that the cache does not have")
    d.call()
    case.table = np.clip(wild, 0, case.pages - 1)
    same(d.result(), case.oracle(), "pages")
    case = U.Attention(34, 4, 2, 64, 64, [3, 4], [100, 128])
    d = DeviceAttention(case)
    d.start.copy_(torch.tensor([-9, 3, 10 ** 9], dtype=torch.int32))
    G.say("attention: starts beyond the rows")
    d.call()
    same(d.result(), case.oracle(), "starts")


@pytest.mark.parametrize("s_dy,o_dy", [((0, 62), (1 << 30, 46)), ((2 ** 31 - 1, 24), (1 << 30, 46)), ((2 ** 31 - 1, 31), (2 ** 31 - 1, 45)), ((2 ** 31 - 1, 32), (1, 0)),
                                       ((2 ** 31 - 1, 33), (-(1 << 30), 45)), ((2 ** 31 - 1, 38), (1 << 30, 47)), ((3, 27), (0, 0)), ((2 ** 31 - 1, 62), (1 << 30, 45))])
def test_attention_of_any_dyadic(gpu, s_dy, o_dy):
    for n, kv in (([1, 1], [90, 700]), ([70, 1], [90, 200])):
        case = U.Attention(35, 3, 1, 64, 64, n, kv)
        case.s_dy, case.o_dy = s_dy, o_dy
        check_attention(case)


def test_attention_of_extreme_values(gpu):
    # -128 in queries and keys, scores at both ends, one key that outweighs all others and ties for the maximum
    for D in (64, 128):
        for n, kv in (([1, 1], [400, 64]), ([100], [300])):
            case = U.Attention(36, 2, 1, D, 64, n, kv)
            case.q[:] = np.where(np.random.default_rng(1).random(case.q.shape) < 0.5, -128, 127)
            case.k[:] = np.where(np.random.default_rng(2).random(case.k.shape) < 0.5, -128, 127)
            check_attention(case)
            case.k[:], case.q[:] = -128, -128
            check_attention(case)


def test_attention_does_not_depend_on_the_batch(gpu):
    # a row alone, among others, and as the last of a prompt's rows
    torch, G, B = libs()
    case = U.Attention(37, 8, 2, 128, 64, [6, 1, 33], [3000, 500, 700])
    d, want = check_attention(case)
    for b in range(3):
        last = int(case.q_start[b + 1]) - 1
        one = U.Attention(37, 8, 2, 128, 64, [6, 1, 33], [3000, 500, 700])
        one.q, one.out = case.q[last:last + 1].copy(), case.out[last:last + 1].copy()
        one.n, one.kv, one.batch, one.rows = np.array([1]), case.kv[b:b + 1], 1, 1
        one.q_start, one.kv_len, one.table = np.array([0, 1], np.int32), case.kv_len[b:b + 1], case.table[b:b + 1]
        e = DeviceAttention(one)
        e.call()
        same(e.result(), want[last:last + 1], "row alone")


def test_attention_of_many_sequences(gpu):
    rng = np.random.default_rng(38)
    kv = rng.integers(0, 150, 700)
    check_attention(U.Attention(38, 2, 1, 64, 64, [1] * 700, kv))
    n = rng.integers(0, 4, 300)
    check_attention(U.Attention(39, 2, 1, 64, 64, n, rng.integers(0, 150, 300)))


@pytest.mark.parametrize("batch,heads,D,window,sinks", [(64, 2, 64, 0, 0), (65, 2, 64, 0, 0), (32, 4, 128, 0, 0), (33, 4, 128, 0, 0), (33, 4, 128, 130, 70), (16, 4, 128, 130, 70)])
def test_attention_on_both_sides_of_a_workgroup_a_unit(gpu, batch, heads, D, window, sinks):
    # two tiles of rows each: 256 workgroups and a few more, ways of no block up to more than twice eight
    rng = np.random.default_rng(batch + D)
    n = rng.integers(0, 18, batch)
    n[0] = 17
    check_attention(U.Attention(40 + batch, heads, heads, D, 64, n, rng.integers(0, 1300, batch), window, sinks))


@pytest.mark.parametrize("n,kv,hq,hk,D,kernel", [
    ([16], [4000], 32, 8, 128, "paged_attention_kernel"), ([4], [4000], 32, 8, 128, "paged_join_kernel"), ([16] * 12, [4000] * 12, 16, 16, 64, "paged_attention_kernel"),
    ([20] * 30, [1000] * 30, 12, 12, 64, "paged_attention_kernel"), ([40] * 30, [1000] * 30, 12, 12, 64, "paged_prompt_kernel"),
    ([5] * 40, [2000] * 40, 32, 8, 128, "paged_prompt_kernel"), ([5] * 40, [600] * 40, 32, 8, 128, "paged_attention_kernel")])
def test_attention_rules_for_few_rows(gpu, n, kv, hq, hk, D, kernel):
    torch, G, B = libs()
    case = U.Attention(61, hq, hk, D, 64, n, kv)
    G.say("attention by rule: %s" % kernel)
    d = DeviceAttention(case)
    d.call()
    d.result()
    assert B.lib().ibert_last_kernel().decode().startswith(kernel)


@pytest.mark.parametrize("n,kv,hq,hk,D,window,sinks,kernel", [
    # one prompt among single rows that take one launch, three, or the scores twice; sequences of no and of two rows among them; a window
    ([1] * 20 + [600] + [1] * 10, [700] * 20 + [600] + [0, 1, 64, 65, 300, 5, 128, 129, 1000, 900], 8, 2, 128, 0, 0, "paged_prompt_kernel"),
    ([1, 0, 2, 1500, 1, 1, 3, 1] + [0] * 12, [9000, 70, 80, 1600, 1, 0, 2, 5000] + [10] * 12, 8, 2, 128, 0, 0, "paged_prompt_kernel"),
    ([1] * 30 + [700] + [1] * 34, [3000] * 30 + [900] + [2500] * 34, 16, 1, 128, 0, 0, "paged_prompt_kernel"),
    ([700] + [1] * 20, [900] + [2100] * 20, 12, 12, 64, 333, 5, "paged_prompt_kernel"),
    ([1] * 24 + [520], [100] * 24 + [520], 24, 4, 64, 0, 0, "paged_prompt_kernel")])
def test_attention_of_single_rows_among_prompts(gpu, n, kv, hq, hk, D, window, sinks, kernel):
    torch, G, B = libs()
    case = U.Attention(70 + hq, hq, hk, D, 64, n, kv, window, sinks, pad=5)
    G.say("single rows among prompts: %d sequences, %d rows" % (case.batch, case.rows))
    d, want = check_attention(case)
    for _ in range(2):
        d.call()
        same(d.result(), want, "out")
    assert B.lib().ibert_last_kernel().decode().startswith(kernel)


def test_attention_of_single_rows_in_a_batch_that_is_mostly_empty(gpu):
    # the single rows' heads are tiles of prompts themselves, and counted; with and without a longer sequence among them
    rng = np.random.default_rng(80)
    for longest in (20, 2):
        n = np.zeros(400, np.int64)
        n[rng.permutation(400)[:30]] = 1
        n[137] = longest
        check_attention(U.Attention(80 + longest, 40, 1, 64, 64, n, rng.integers(0, 200, 400)), max_q=20)


# ------------------------------------------------------------------------------------------- graphs and streams
def test_decoder_calls_in_graphs_and_on_another_stream(gpu):
    torch, G, B = libs()
    cases = [U.Attention(40, 8, 2, 128, 64, [1, 1], [5000, 77]), U.Attention(41, 4, 4, 64, 64, [70, 5], [90, 300]), U.Attention(42, 12, 12, 64, 64, [1] * 3, [10, 64, 200]),
             U.Attention(45, 4, 1, 64, 64, [1] * 64, [4500] * 64)]          # (the last: more LDS than a launch has by itself)
    devs = [DeviceAttention(c) for c in cases]
    pages = DevicePages(U.Pages(43, *U.mixed_lengths(np.random.default_rng(43), 70, 300), 64))
    rot = U.Rotary(44, 40, 4, 2, 64, 64, False, 64, True, True)
    tk, tv, tq, tx, tc, tp, ts, gq, gk = (G.to_dev(a) for a in (rot.k0, rot.v0, rot.q0, rot.qkv, rot.cs, rot.positions, rot.slots, rot.gq, rot.gk))
    desc, cache = rot.descs(tk, tv)
    want, rot_want = [c.oracle() for c in cases], rot.oracle()

    def everything(stream=None):
        for d in devs:
            d.call(stream)
        pages.call(stream)
        B.ibert_rotary_append_i(desc, cache, tx, rot.qkv.shape[1], tc, tp, ts, gq, gk, rot.rows, tq, rot.q0.shape[1], stream)

    def check():
        torch.cuda.synchronize()
        for d, w in zip(devs, want):
            same(d.result(), w, "out")
            d.out[:-64].fill_(5)
            d.out[:-64].view(w.shape).copy_(torch.from_numpy(d.case.out))
        pages.check()
        for got, w, what in zip((tq, tk, tv), rot_want, "qkv"):
            same(got, w, what)
        tq.copy_(torch.from_numpy(rot.q0))
        tk.copy_(torch.from_numpy(rot.k0))
        tv.copy_(torch.from_numpy(rot.v0))
        for t in pages.o.values():
            t.fill_(77)
    G.say("decoder calls: eager")
    everything()
    check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    G.say("decoder calls: another stream, named")
    everything(side)
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        everything()
    for k in range(4):
        G.say("decoder calls: replay %d" % k)
        graph.replay()
        check()
        everything()
        check()
    # a replay takes the lengths that stand there now
    devs[0].kv.copy_(torch.tensor([3000, 64], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    cases[0].kv_len[:] = (3000, 64)
    same(devs[0].result(), cases[0].oracle(), "after other lengths")


def test_attention_at_the_largest_batch_and_bound_of_rows(gpu):
    # 65535 sequences, most of them empty, in every form; 65535 tiles of 64 rows as the bound of a few, with starts (tiles are counted) and without
    n, kv = np.ones(65535, np.int64), np.zeros(65535, np.int64)
    kv[[0, 1, 511, 512, 40000, 65533, 65534]] = (64, 1, 65, 300, 128, 7, 200)
    check_attention(U.Attention(95, 2, 1, 64, 64, n, kv))
    n[[3, 65534]], n[100:200] = (0, 70), 0
    check_attention(U.Attention(96, 2, 1, 64, 64, n, kv))
    case = U.Attention(97, 1, 1, 64, 64, [1, 70, 1], [200, 130, 64])
    check_attention(case, max_q=64 * 65535)
    check_attention(U.Attention(98, 2, 1, 64, 64, [1, 1], [70, 1]), plain_rows=True, max_q=32 * 65535)
    check_attention(U.Attention(99, 1024, 1024, 64, 64, [1, 20], [70, 130]))


def test_attention_under_bounds_far_above_the_lengths(gpu):
    # what a captured step hands over: the longest context and the most rows that may come
    for n, kv, hq, hk, D, max_q in (([1] * 3, [70, 0, 4000], 8, 2, 128, 1), ([1, 3, 1], [700, 64, 5], 4, 4, 64, 16), ([1] * 40, [100] * 39 + [9000], 16, 16, 64, 1), ([90, 1], [100, 2], 8, 2, 128, 2048)):
        check_attention(U.Attention(87 + D, hq, hk, D, 128, n, kv, pad=max_q), max_q=max_q, max_kv=131072)
    # without starts every sequence has one row, whatever the bound says
    check_attention(U.Attention(88, 8, 2, 128, 64, [1] * 20, [700] * 19 + [65], pad=9), plain_rows=True, max_q=600, max_kv=5000)


def test_decoder_calls_on_two_streams_at_once(gpu):
    # a workspace, page tables and cache for each; keys split on both, single rows beside a prompt on one of them
    torch, G, B = libs()
    sides = [torch.cuda.Stream() for _ in range(2)]
    cases = [U.Attention(89, 8, 2, 128, 64, [1, 1], [9000, 700]), U.Attention(90, 16, 4, 128, 64, [1, 1, 600, 1], [9000, 3000, 650, 300])]
    pages = [U.Pages(91 + i, *U.mixed_lengths(np.random.default_rng(91 + i), 300, 900), 64) for i in range(2)]
    want = [c.oracle() for c in cases]
    devs, tables = [DeviceAttention(c) for c in cases], [[DevicePages(p) for _ in range(6)] for p in pages]
    assert all(d.size > 0 for d in devs)
    torch.cuda.synchronize()
    G.say("decoder calls on two streams")
    for k in range(6):
        for d, t, s in zip(devs, tables, sides):
            t[k].call(s)
            for _ in range(3):
                d.call(s)
    for d, w in zip(devs, want):
        same(d.result(), w, "out")
    for t in tables:
        for p in t:
            p.check()


def test_single_rows_among_prompts_in_a_graph(gpu):
    # two plans in one call, and lengths that change between replays: the same launches then take other rows
    torch, G, B = libs()
    case = U.Attention(93, 16, 4, 128, 64, [1, 1, 600, 1], [9000, 3000, 650, 300], pad=40)
    rot = U.Rotary(94, 100, 5, 5, 128, 128, True, 64, True, True, 16, range(90, 100))
    tk, tv, tq, tx, tc, tp, ts, gq, gk = (G.to_dev(a) for a in (rot.k0, rot.v0, rot.q0, rot.qkv, rot.cs, rot.positions, rot.slots, rot.gq, rot.gk))
    desc, cache = rot.descs(tk, tv)
    d = DeviceAttention(case)
    assert d.size > 0
    B.ibert_rotary_override(2)
    try:
        graph = torch.cuda.CUDAGraph()
        d.call()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            d.call()
            B.ibert_rotary_append_i(desc, cache, tx, rot.qkv.shape[1], tc, tp, ts, gq, gk, rot.rows, tq, rot.q0.shape[1])
    finally:
        B.ibert_rotary_override(-1)
    rot_want = rot.oracle()
    for k, (n, kv) in enumerate([(case.n, case.kv), ([2, 1, 599, 1], [8999, 1, 9000, 64]), ([1] * 4, [2000, 0, 5000, 77]), ([0, 600, 1, 40], [5, 600, 8000, 39])]):
        case.n, case.kv = np.array(n), np.array(kv)
        case.q_start, case.kv_len = np.concatenate([[0], np.cumsum(n)]).astype(np.int32), np.array(kv, np.int32)
        for _ in range(2):
            G.say("single rows among prompts, replay %d" % k)
            d.start.copy_(torch.from_numpy(case.q_start))
            d.kv.copy_(torch.from_numpy(case.kv_len))
            d.out[:-64].copy_(torch.from_numpy(case.out.reshape(-1)))
            d.ws.fill_(-1)
            for t, old in ((tq, rot.q0), (tk, rot.k0), (tv, rot.v0)):
                t.copy_(torch.from_numpy(old))
            graph.replay()
            same(d.result(), case.oracle(), "out of replay %d" % k)
            for got, w, what in zip((tq, tk, tv), rot_want, "qkv"):
                same(got, w, what)


# ------------------------------------------------------------------------------------------- as a decoder runs them
@pytest.mark.parametrize("hq,hk,D,R,inter,norm,window,sinks", [(12, 12, 64, 64, False, False, 0, 0), (8, 2, 128, 64, True, True, 100, 4)])
def test_a_decoder_layer_step_by_step(gpu, hq, hk, D, R, inter, norm, window, sinks):
    """QKV projection, page tables, rotation + append and attention of prompts and of the tokens after them, with sequences that
    come, go and wait for pages, against the oracle's chain of the same steps."""
    torch, G, B = libs()
    rng = np.random.default_rng(50)
    H, page, width, num, rows, batch, max_pos = 256, 64, 6, 14, 260, 4, 400
    heads = hq + 2 * hk
    w = rng.integers(-127, 128, (heads * D, H)).astype(np.int8)
    bias = rng.integers(-1000, 1000, heads * D).astype(np.int32)
    mult, shift = B.ibert_channel_dyadics_from_scales(1.0, np.full(heads * D, 32 / (30 * 73 * 16.0)), 1.0)
    freqs = B.ibert_rotary_freqs(B.RotaryScaling(10000.0, 1.0, 1.0, 0.0, 1.0, B.ROPE_NONE), R)
    cs = B.ibert_rotary_table_from_freqs(freqs, max_pos)
    g, gs = B.ibert_head_norm_from_float(rng.normal(1, 0.1, D), 2.0 ** -12)
    dy = U.dyadic(127 / 4 / 4096 / 16384) if norm else U.dyadic(0.9 / 16384)
    s_qk = 4.0 / 127
    att = B.ibert_paged_attention_from_scales(s_qk, s_qk, 1.0, 0.5, D, hq, window, sinks)
    rot = B.RotaryDesc(hq, R, B.ROTARY_INTERLEAVED if inter else B.ROTARY_HALF, max_pos, B.Dyadic(*dy), B.Dyadic(*dy), B.Dyadic(*U.dyadic(0.8)), gs, gs)
    o_rot = oracle.RotaryT(hq, hk, D, page, R, int(inter), max_pos, num, *dy, *dy, *U.dyadic(0.8), gs, gs)
    o_att = oracle.PagedT(hq, hk, D, page, num, width, window, sinks, *att.scores_dy.tuple(), *att.out_dy.tuple())
    cells = num * page * hk * D
    k, v = np.zeros(cells, np.int8), np.zeros(cells, np.int8)
    ring, state, lens, table = rng.permutation(num).astype(np.int32), np.array([0, num], np.int32), np.zeros(batch, np.int32), np.zeros((batch, width), np.int32)
    tk, tv = G.to_dev(k), G.to_dev(v)
    cache = B.KvCache(tk.data_ptr(), tv.data_ptr(), hk, D, page, num)
    t_w, t_b, t_m, t_s, t_cs, t_g, t_ring, t_table = (G.to_dev(a) for a in (w, bias, mult, shift, cs, g, ring, table))
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=G.DEV)       # noqa: E731
    t_state, t_lens = [G.to_dev(np.append(state, 0).astype(np.int32)), i32(3)], [i32(batch), i32(batch)]
    t_start, t_slots, t_pos = i32(batch + 1), i32(rows), i32(rows)
    t_qkv, t_q, t_out = (torch.zeros(rows, n, dtype=torch.int8, device=G.DEV) for n in (heads * D, hq * D, hq * D))
    ws = torch.empty(max(256, B.ibert_paged_attention_workspace_bytes(att, cache, batch, rows, rows, width * page)), dtype=torch.uint8, device=G.DEV)
    d = B.GemmDesc()
    d.M, d.N, d.K, d.batch_outer, d.batch_inner, d.lda, d.ldw, d.ldc = rows, heads * D, H, 1, 1, H, H, heads * D
    d.per_channel, d.out_dtype, d.out_clamp = 1, B.I8, 127
    q, out = np.zeros((rows, hq * D), np.int8), np.zeros((rows, hq * D), np.int8)
    refused = 0
    for step, more in enumerate([(100, 130, 20, 0), (1, 1, 1, 0), (1, 1, 1, 230), (1, -131, 1, 230), (1, 0, 1, 1), (140, 3, 2, 1), (-50, 64, 300, 1)]):
        after = np.maximum(0, lens + np.array(more)).astype(np.int32)
        x = U.normal8(rng, 30, rows, H)
        # the oracle's step
        o = oracle.page_tables(lens, after, page, state, ring, table, rows)
        ring, state, table = o["ring"], o["ring_out"], o["table"]
        refused += int(state[2])
        og = oracle.GemmT(**dict(M=rows, N=heads * D, K=H, batch_outer=1, batch_inner=1, lda=H, ldw=H, ldc=heads * D, per_channel=1, out_dtype=oracle.I8, out_clamp=127))
        qkv = oracle_gemm(og, x, w, bias, mult, shift).reshape(rows, heads * D)
        q, k, v = oracle.rotary_append(o_rot, qkv, cs, o["positions"], o["slots"], g if norm else None, g if norm else None, q, k, v)
        out = oracle.paged_attention(o_att, q, k, v, table, o["q_start"], o["kv_len"], out)
        # the library's
        G.say("decoder step %d" % step)
        B.ibert_page_tables_i(t_lens[step % 2], G.to_dev(after), batch, page, num, t_state[step % 2], t_ring, t_state[1 - step % 2], t_table, width, rows, t_start,
                              t_lens[1 - step % 2], t_slots, t_pos)
        B.ibert_gemm_i8_requant(d, G.to_dev(x), t_w, t_b, t_m, t_s, None, t_qkv)
        B.ibert_rotary_append_i(rot, cache, t_qkv, heads * D, t_cs, t_pos, t_slots, t_g if norm else None, t_g if norm else None, rows, t_q, hq * D)
        B.ibert_paged_attention_i(att, cache, t_q, hq * D, t_table, width, t_start, t_lens[1 - step % 2], batch, rows, rows, width * page, t_out, hq * D, ws)
        torch.cuda.synchronize()
        same(t_qkv, qkv, "qkv of step %d" % step)
        for got, want, what in ((t_q, q, "q"), (tk, k, "k"), (tv, v, "v"), (t_out, out, "out"), (t_table, table, "table"), (t_ring, ring, "ring")):
            same(got, want, "%s of step %d" % (what, step))
        lens = o["kv_len"]
    assert refused > 0 and out.any()


def oracle_gemm(desc, x, w, bias, mult, shift):
    out = np.zeros(desc.M * desc.N, np.int8)
    rc = oracle.lib().orc_gemm_requant(oracle.C.byref(desc), x.ctypes.data, w.ctypes.data, bias.ctypes.data, mult.ctypes.data, shift.ctypes.data, None, out.ctypes.data)
    assert rc == 0
    return out
