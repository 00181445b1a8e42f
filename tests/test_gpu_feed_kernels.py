"""The kernels that the rules pick for serving sizes: the logits' slices and their sums of biases, tiles of many channels, the persistent gated block's
shares of the XCDs, sums at the ends of their bits.  Bit for bit against the definitions in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import feed_util as U
from test_gpu_decoder import libs, same
from test_gpu_feed import DeviceLogits, ran, run


# ------------------------------------------------------------------------------------------- logits
def check_logits(c, kernel, what, off=0, in_place=False):
    torch, G, B = libs()
    G.say("logits: %s, at %d%s" % (what, off, ", in place" if in_place else ""))
    d = DeviceLogits(c, off, in_place)
    d.call()
    torch.cuda.synchronize()
    ran("logits_adjust_kernel<%d>" % kernel)
    if in_place:
        same(d.x, U.logits_by_rows(c, c.x), what)
    else:
        same(d.y[:c.y0.size], U.logits_by_rows(c), what)
        assert bool((d.y[c.y0.size:] == 77).all()), "wrote past the end: " + what


def wide_values(seed, n):
    """Biases of which a few take a row's sums beyond 32 bits."""
    rng = np.random.default_rng(seed)
    v = rng.integers(-500, 500, n).astype(np.int32)
    v[rng.random(n) < 0.02] = U.LOW
    v[rng.random(n) < 0.02] = U.HIGH
    return v


# rows x vocabulary whose slices have 2048 or 4096 tokens; ends of a slice, of half a slice and of neither; 16-byte rows and others
SLICED = [(3, 1030, 2048), (2, 2048, 2048), (5, 5121, 2048), (2, 7000, 2048), (64, 33000, 4096), (130, 16388, 4096), (136, 17001, 4096), (128, 14336, 4096)]


@pytest.mark.parametrize("rows,vocab,kernel", SLICED)
def test_logits_sums_of_biases_beyond_32_bits(gpu, rows, vocab, kernel):
    rng = np.random.default_rng(vocab)
    for off, in_place in ((0, False), (1, False), (0, True)):
        blens = rng.integers(0, 700, rows)
        blens[0], blens[-1] = 1500, 3
        c = U.Logits(vocab, rng.integers(0, 300, rows), vocab, blens, 3)
        c.values[:] = wide_values(vocab, c.values.size)
        c.ids[:40] = rng.integers(0, vocab)               # forty of one token, whose sum passes 32 bits on the way
        c.values[:40:2], c.values[1:40:2] = U.LOW, U.HIGH
        check_logits(c, kernel, "%d x %d, wide biases" % (rows, vocab), off, in_place)


def test_logits_a_long_list_of_biases_is_gone_through_a_fixed_number_of_times(gpu):
    # one value beyond 2^31 / n among n = 60000: once more for each half of a slice, where a walk for every token it holds would take the list's length squared
    torch, G, B = libs()
    rows, vocab, n = 4, 30000, 60000
    c = U.Logits(1, [100] * rows, vocab, [n] * rows, 2)
    c.values[:] = np.random.default_rng(2).integers(-500, 500, c.values.size)
    times = []
    for ban in (False, True):
        if ban:
            c.values[c.bstart[:-1] + 5] = U.LOW
            c.ids[c.bstart[:-1] + 5] = 77
        check_logits(c, 2048, "60000 biases a row%s" % (", one token banned" if ban else ""))
        d = DeviceLogits(c)
        best = 1e9
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                d.call()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
    assert times[1] < 8 * times[0], times             # (three walks for one, and beside them the same work)


@pytest.mark.parametrize("rows,vocab,kernel", SLICED + [(70, 33000, 4096)])
def test_logits_slices(gpu, rows, vocab, kernel):
    # histories, biases whose sums have 32 bits, masks; rows dealt to the XCDs (a multiple of eight, 128 and more) or not
    rng = np.random.default_rng(rows)
    lens, blens = rng.integers(0, 400, rows), rng.integers(0, 300, rows)
    lens[0], lens[-1], blens[-1] = 9000, 0, 0
    c = U.Logits(vocab + 1, lens, vocab, blens, 4)
    c.values[:] = rng.integers(-700, 700, c.values.size)
    for off, in_place in ((0, False), (2, False), (0, True)):
        check_logits(c, kernel, "%d x %d" % (rows, vocab), off, in_place)
    c = U.Logits(vocab + 2, lens, vocab, None, 0, (5, 3, 0))
    check_logits(c, kernel, "%d x %d, strides, histories alone" % (rows, vocab))


@pytest.mark.parametrize("rows,vocab,kernel", [(12, 5000, 2048), (72, 30000, 4096)])
def test_logits_biases_on_both_sides_of_the_32_bit_line(gpu, rows, vocab, kernel):
    # lists of n equal values for one token: (2^31 - 1) / n still has sums of 32 bits, one more in size has not
    lens = [(1, 7, 1000)[r // 4 % 3] for r in range(rows)]
    c = U.Logits(3, [20] * rows, vocab, lens, 0)
    for r, n in enumerate(lens):
        small = (2 ** 31 - 1) // n
        c.values[c.bstart[r]:c.bstart[r + 1]] = (small, min(small + 1, U.HIGH), -small, -small - 1)[r % 4]
        t = int(np.random.default_rng(r).integers(0, vocab))
        c.ids[c.bstart[r]:c.bstart[r + 1]] = t
        c.x[r, t] = (-5, 5, 5, -5)[r % 4]
    check_logits(c, kernel, "biases at the line")


# ------------------------------------------------------------------------------------------- few rows
SHAPES = [(1, 1, 1), (1, 17, 15), (2, 33, 129), (5, 100, 304), (8, 64, 2048), (17, 130, 512), (33, 96, 1000), (64, 48, 640), (65, 341, 768), (130, 70, 128)]


@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("form", [(2, 1), (2, 4)], ids=["8_rows", "32_rows"])
def test_w4_two_tiles_of_channels(gpu, form, group, zeros):
    from paper_2101_01321_amd import binding as B
    B.ibert_rows_override(*form)
    try:
        for M, N, K in SHAPES:
            run(U.Rows4(M + N, M, N, K, group, zeros, ("i8", "i16", "i32")[(M + N) % 3], residual=bool(N % 2), bias=M % 3 != 0), "w4 %d x %d x %d, groups of %d" % (M, N, K, group))
            if K % 16 == 0:
                ran("rows_ring_kernel<true, %d, 2," % form[1])
            if form == (2, 4):
                run(U.Gated(M + N, M, N, K, M % 2, group, zeros), "w4 gated %d x %d x %d, groups of %d" % (M, N, K, group))
                if K % 16 == 0:
                    ran("rows_ring_kernel<true, 4, 4,")
    finally:
        B.ibert_rows_override(-1, -1)


# what serving calls, small in K: heads of many channels, batches
PICKED = [("w4", 1, 24600, 144, "<true, 1, 2,"), ("w4", 8, 30011, 128, "<true, 1, 2,"), ("w4", 13, 24600, 256, "<true, 2, 2,"), ("w4", 40, 4099, 272, "<true, 4, 2,"),
          ("w4", 130, 6600, 2048, "<true, 4, 4,"), ("w4", 64, 8200, 8192, "<true, 4, 4,"), ("gated", 130, 3300, 144, "<true, 4, 4,"), ("gated", 64, 8200, 256, "<true, 4, 4,")]


@pytest.mark.parametrize("kind,M,N,K,kernel", PICKED)
def test_w4_kernels_that_the_rule_picks(gpu, kind, M, N, K, kernel):
    for group, zeros in ((128, False), (32, True)):
        if kind == "w4":
            run(U.Rows4(M, M, N, K, group, zeros, "i32" if M < 16 else "i16", residual=M >= 16), "w4 %d x %d x %d by the rule" % (M, N, K))
        else:
            run(U.Gated(M, M, N, K, M % 3 // 2, group, zeros), "w4 gated %d x %d x %d by the rule" % (M, N, K))
        ran("rows_ring_kernel" + kernel)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_sums_of_the_longest_runs_in_32_bits(gpu, group, zeros):
    # 32 chunks of K to a wavefront, every product at its largest: 4096 * 128 * 15 * 255 < 2^31; one chunk more is the other kernel's
    for K, kernel in ((32768, "rows_ring_kernel"), (32784, "rows_any_kernel")):
        for M in (1, 20):
            c = U.Rows4(K, M, 20, K, group, zeros, "i32", extreme=True)
            c.ch.m[:], c.ch.s[:] = 1 << 30, 36            # (nothing is cut off here but by INT32 itself)
            c.a[-1] = 1
            c.acc = np.clip(U.product(c.a, c.w4.whole()) + c.ch.bias(), U.LOW, U.HIGH)
            run(c, "w4 extreme, groups of %d, K %d" % (group, K))
            ran(kernel)
            c = U.Rows4(K + 1, M, 20, K, group, zeros, "i32", extreme=True)
            # signs in turn from run to run of 4096: every run's sum is at an end of its 32 bits, what they come to is small
            c.a[:, :K] = np.where(np.arange(K) // 4096 % 2 == 0, -128, 127)
            c.a[:, K - 4096:] = 3
            c.ch.m[:], c.ch.s[:] = 1 << 30, 31
            acc = U.product(c.a, c.w4.whole()) + c.ch.bias()
            c.acc = np.clip(acc, U.LOW, U.HIGH)
            run(c, "w4 runs of both signs, groups of %d, K %d" % (group, K))
            ran(kernel)


# ------------------------------------------------------------------------------------------- many tokens
@pytest.fixture(params=[0, 1, 3], ids=["tall", "low", "narrow"])
def persistent(request, gpu):
    from paper_2101_01321_amd import binding as B
    B.ibert_rows_override(0, request.param)
    yield request.param
    B.ibert_rows_override(-1, -1)


@pytest.mark.parametrize("act", [0, 1], ids=["silu", "gelu"])
def test_persistent_gated_columns_dealt_to_four_groups_of_xcds(persistent, act):
    # columns of tiles a multiple of four, more than 4 MB of weights, eight rows of tiles and more
    run(U.Gated(act, 2100, 2048, 1040, act), "persistent gated, 4.3 MB of weights")
    ran("gated_stream_kernel")


def test_persistent_gated_gelu_beyond_where_erf_is_one(persistent):
    # gates on both sides of -q_b, where erf is cut off; its table has no room in the narrow tile, whose kernel computes it
    from paper_2101_01321_amd import binding as B
    for name in ("by hand", "from a scale"):
        c = U.Gated(21, 700, 300, 256, B.GATE_GELU)
        if name == "by hand":
            c.params.gelu = B.GeluParams(-1000, -500000, -400000, (2 ** 31 - 1) // 900000, B.Dyadic(-(1 << 30), 46))
        else:
            c.params = B.ibert_gate_params_from_scales(B.GATE_GELU, 1 / 390, 1 / 2000, 1 / 16)
        q_b, q_max = c.params.gelu.q_b, c.params.gelu.q_max
        assert -1700 < q_b <= -896 and q_max > -q_b
        c.ch.m[:300], c.ch.s[:300] = c.ch.m[:300], c.ch.s[:300] - 2        # gates four times as large
        run(c, "persistent gated, gates beyond -q_b, constants " + name)
        g = U.dy(c.acc[:, :300], c.ch.m[:300], c.ch.s[:300])
        assert (np.abs(g) > -q_b).mean() > 0.05 and (np.abs(g) < -q_b).mean() > 0.05 and (np.abs(g) > q_max).any()
        assert np.unique(c.expected()).size > 100
        ran("gated_stream_kernel<%d" % (0 if persistent == 3 else 2))


# ------------------------------------------------------------------------------------------- the ends of what the calls take
def strided(values, ld, fill=0):
    """A [rows, n] int8 array as rows ld bytes apart on the GPU: the whole buffer and the view of its rows."""
    torch, G, B = libs()
    rows, n = values.shape
    whole = torch.full((rows * ld,), fill, dtype=torch.int8, device=G.DEV)
    view = whole.view(rows, ld)[:, :n]
    view.copy_(torch.from_numpy(np.ascontiguousarray(values)).to(G.DEV))
    return whole, view


@pytest.mark.parametrize("M,F,K,lda,ldw,ldc,kernel", [
    (40, 70, 144, 1 << 24, 1 << 26, 1 << 27, "rows_ring_kernel"), (300, 70, 150, (1 << 24) + 1, (1 << 26) + 16, (1 << 24) + 3, "rows_any_kernel"),
    (4500, 2200, 144, (1 << 20) - 16, (1 << 20) - 16, (1 << 20) - 16, "gated_stream_kernel")])
def test_i8_gated_offsets_beyond_32_bits(gpu, M, F, K, lda, ldw, ldc, kernel):
    torch, G, B = libs()
    c = U.Gated(M, M, F, K, M % 2)
    G.say("i8 gated %d x %d x %d, leading dimensions %d, %d, %d" % (M, F, K, lda, ldw, ldc))
    a, w = strided(c.a, lda)[0], strided(c.w, ldw)[0]
    out, rows = strided(c.c0, ldc, 77)
    desc = c.desc()
    desc.lda, desc.ldw, desc.ldc = lda, ldw, ldc
    B.ibert_gemm_i8_gated(desc, a, w, G.to_dev(c.ch.b), G.to_dev(c.ch.m), G.to_dev(c.ch.s), out)
    torch.cuda.synchronize()
    ran(kernel)
    same(rows, c.expected(), "offsets beyond 32 bits")
    rows.fill_(77)
    assert all(bool((x == 77).all()) for x in out.split(1 << 30)), "wrote between the rows"


@pytest.mark.parametrize("K,lda,kernel", [(144, 1 << 24, "rows_ring_kernel"), (150, (1 << 24) + 3, "rows_any_kernel")])
def test_w4_offsets_beyond_32_bits(gpu, K, lda, kernel):
    torch, G, B = libs()
    M, N, ldc = 300, 40, (1 << 24) + 5
    c = U.Rows4(K, M, N, K, 64, True, "i8", residual=True)
    G.say("w4 %d x %d x %d, leading dimensions %d, %d" % (M, N, K, lda, ldc))
    a, r = strided(c.a, lda)[0], strided(c.r, ldc)[0]
    out, rows = strided(c.c0, ldc, 77)
    t = [G.to_dev(x) for x in c.w4.pack()]
    desc = c.desc()
    desc.lda, desc.ldc, desc.ldr = lda, ldc, ldc
    B.ibert_gemm_w4_requant(desc, a, B.W4Weights(t[0].data_ptr(), t[1].data_ptr(), t[2].data_ptr(), 64), G.to_dev(c.ch.b), G.to_dev(c.ch.m), G.to_dev(c.ch.s), r, out)
    torch.cuda.synchronize()
    ran(kernel)
    same(rows, c.expected(), "offsets beyond 32 bits")
    rows.fill_(77)
    assert all(bool((x == 77).all()) for x in out.split(1 << 30)), "wrote between the rows"


@pytest.mark.parametrize("out", ["i16", "i32"])
def test_w4_results_at_odd_addresses(gpu, out):
    torch, G, B = libs()
    from test_gpu_feed import OnDevice
    for M, N, K in ((3, 37, 144), (20, 70, 150)):
        c = U.Rows4(M, M, N, K, 32, False, out, ld=(0, 3, 0))
        d = OnDevice(c)
        size = c.c0.nbytes
        for off in (1, 2, 3):
            G.say("w4, %s at %d bytes" % (out, off))
            room = torch.full((size + 16,), 77, dtype=torch.uint8, device=G.DEV)
            room[off:off + size] = torch.from_numpy(c.c0.reshape(-1).view(np.uint8)).to(G.DEV)
            d.out = room[off:]
            d.call()
            torch.cuda.synchronize()
            got = room.cpu().numpy()
            assert np.array_equal(got[off:off + size].view(c.dtype), c.expected().reshape(-1)) and (got[:off] == 77).all() and (got[off + size:] == 77).all()


def test_logits_of_the_largest_vocabulary(gpu):
    torch, G, B = libs()
    rows, vocab = 1, 1 << 26
    c = U.Logits(5, [3000], vocab, [400])
    G.say("logits, %d x %d" % (rows, vocab))
    c.tokens[:5], c.ids[:5] = (vocab - 1, 0, vocab - 1, vocab, 4096), (vocab - 1, vocab - 1, 0, vocab, 4095)
    check_logits(c, 4096, "the largest vocabulary")


def test_logits_rows_of_two_slices_that_no_launch_holds(gpu):
    # 2^21 rows of two slices; 34 GB in place, so that rows pass 2^32 elements too
    torch, G, B = libs()
    rows, vocab = (1 << 21) + 9, 4097
    G.say("logits, %d rows of %d" % (rows, vocab))
    x = torch.zeros(rows * vocab, dtype=torch.int32, device=G.DEV)
    x[-1], x[0] = U.LOW, -3
    params = torch.tensor([1, 0, 1, 0, 5, 7, -1], dtype=torch.int32, device=G.DEV).repeat(rows, 1)
    first = torch.zeros(rows + 1, dtype=torch.int32, device=G.DEV)
    tokens = torch.tensor([4096, 0, 0, 4096, 2, 4096, 17], dtype=torch.int32, device=G.DEV)
    # row 0: [4096, 0, 0]; the last of the first launch: [4096, 2]; the last: [4096, 17]
    first[1:], first[1 << 21:], first[rows:] = 3, 5, 7
    B.ibert_logits_adjust_i(B.LogitsDesc(rows, vocab, vocab, vocab, 7, 0, 0, 0), x, params, tokens, first, first, None, None, None, None, x)
    torch.cuda.synchronize()
    ran("logits_adjust_kernel<4096>")
    r = (1 << 21) - 1
    want = {0: -3 - 5 - 14, 4096: -12, r * vocab + 2: -12, r * vocab + 4096: -12, (rows - 1) * vocab + 17: -12, rows * vocab - 1: U.LOW}
    for at, v in want.items():
        assert int(x[at]) == v, at
        x[at] = 0
    assert not any(bool(y.any()) for y in x.split(1 << 30))
