"""The gated block, the products with 4-bit weights and the logits' adjustment on the GPU against their definitions in 64 bits, bit for bit, and a
decoder's feed-forward and head run through them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import feed_util as U
from test_gpu_decoder import libs, same


@pytest.fixture(params=[(-1, -1), (1, 0), (0, 0), (0, 1), (1, 1), (1, 4), (2, 2), (2, 8), (4, 1), (4, 4)], ids=lambda p: "t%d_g%d" % p)
def form(request, gpu):
    from paper_2101_01321_amd import binding as B
    B.ibert_rows_override(*request.param)
    yield request.param
    B.ibert_rows_override(-1, -1)


def moved(t, off):
    """t behind `off` elements of its own buffer."""
    import torch
    if off == 0:
        return t
    room = torch.zeros(t.numel() + off, dtype=t.dtype, device=t.device)
    room[off:] = t.reshape(-1)
    return room[off:]


class OnDevice:
    """The tensors of a U.Gated or U.Rows4; guard rows behind the output."""

    def __init__(self, c, off=0):
        torch, G, B = libs()
        self.c, dev = c, G.to_dev
        self.a = moved(dev(c.a), off)
        self.m, self.s = dev(c.ch.m), dev(c.ch.s)
        self.b = None if c.ch.b is None else dev(c.ch.b)
        self.keep = []
        if isinstance(c, U.Gated) and c.group is None:
            self.w = moved(dev(c.w), off)
        elif isinstance(c, U.Gated):
            self.g, self.u = self.weights(c.g4), self.weights(c.u4)
        else:
            self.w = self.weights(c.w4)
            self.r = None if c.r is None else moved(dev(c.r), off)
        self.guard = 3 * c.c0.shape[1]
        full = np.concatenate([c.c0.reshape(-1), np.full(self.guard, 77, c.c0.dtype)])
        self.out = moved(dev(full), off)

    def weights(self, w4):
        torch, G, B = libs()
        t = [None if x is None else G.to_dev(x) for x in w4.pack()]
        self.keep.append(t)
        return B.W4Weights(t[0].data_ptr(), t[1].data_ptr(), None if t[2] is None else t[2].data_ptr(), w4.group)

    def call(self, stream=None):
        torch, G, B = libs()
        c = self.c
        if isinstance(c, U.Rows4):
            B.ibert_gemm_w4_requant(c.desc(), self.a, self.w, self.b, self.m, self.s, self.r, self.out, stream)
        elif c.group is None:
            B.ibert_gemm_i8_gated(c.desc(), self.a, self.w, self.b, self.m, self.s, self.out, stream)
        else:
            B.ibert_gemm_w4_gated(c.desc(), self.a, self.g, self.u, self.b, self.m, self.s, self.out, stream)

    def check(self, what):
        n = self.out.numel() - self.guard
        same(self.out[:n], self.c.expected(), what)
        assert bool((self.out[n:] == 77).all()), "wrote past the end of the output: " + what


def run(c, what, off=0):
    torch, G, B = libs()
    G.say(what)
    d = OnDevice(c, off)
    d.call()
    torch.cuda.synchronize()
    d.check(what)


GATED = [(1, 1, 1), (1, 16, 128), (1, 17, 15), (2, 33, 129), (5, 100, 300), (16, 64, 256), (17, 130, 512), (33, 96, 1000), (64, 48, 640), (65, 341, 768), (130, 70, 128)]


@pytest.mark.parametrize("act", [0, 1], ids=["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", GATED)
def test_i8_gated(form, M, F, K, act):
    run(U.Gated(M + F + K, M, F, K, act), "i8 gated %d x %d x %d" % (M, F, K))


@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("M,F,K", GATED)
def test_w4_gated(form, M, F, K, group, zeros):
    run(U.Gated(M + F + K, M, F, K, (M + group // 32) % 2, group, zeros), "w4 gated %d x %d x %d, groups of %d" % (M, F, K, group))


@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("M,N,K", GATED + [(3, 40, 9000), (40, 600, 5000)])
def test_w4(form, M, N, K, group, zeros):
    out = ("i8", "i16", "i32")[(M + N + group // 32) % 3]
    run(U.Rows4(M + N + K, M, N, K, group, zeros, out, residual=bool((N + zeros) % 2), bias=M % 3 != 0), "w4 %d x %d x %d, groups of %d, %s" % (M, N, K, group, out))


@pytest.fixture(params=[0, 1, 3], ids=["tall", "low", "narrow"])
def persistent(request, gpu):
    from paper_2101_01321_amd import binding as B
    B.ibert_rows_override(0, request.param)
    yield
    B.ibert_rows_override(-1, -1)


def ran(kernel):
    from paper_2101_01321_amd import binding as B
    assert B.lib().ibert_last_kernel().decode().startswith(kernel), B.lib().ibert_last_kernel()


@pytest.mark.parametrize("act", [0, 1], ids=["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", [(256, 128, 128), (257, 129, 256), (300, 400, 384), (1000, 127, 1024), (511, 1, 256), (5150, 2050, 128), (4100, 4096, 384), (9000, 1300, 256), (300, 130, 16), (300, 130, 112), (700, 257, 144), (5000, 1500, 272), (2000, 400, 1040)])
def test_persistent_gated(persistent, M, F, K, act):
    # ragged tokens and channels; up to two tiles and more to a workgroup, columns shared by XCDs or not
    run(U.Gated(M + F + K + act, M, F, K, act), "persistent gated %d x %d x %d" % (M, F, K))
    ran("gated_stream_kernel")


@pytest.mark.parametrize("act", [0, 1], ids=["silu", "gelu"])
@pytest.mark.parametrize("ld,off", [((16, 32, 16), 0), ((0, 0, 3), 0), ((0, 0, 8), 16), ((112, 0, 16), 16)])
def test_persistent_gated_strides(persistent, ld, off, act):
    run(U.Gated(act, 290, 200, 256, act, ld=ld), "persistent gated, strides %s, at %d" % (ld, off), off)
    ran("gated_stream_kernel")


@pytest.mark.parametrize("act", [0, 1], ids=["silu", "gelu"])
def test_persistent_gated_any_constants(persistent, act):
    from paper_2101_01321_amd import binding as B
    # shifts below 33, biases of 31 bits and an output shift below 33 take the general epilogue, tile by tile; the tiles beside them do not
    c = U.Gated(7 + act, 5000, 1400, 128, act)
    c.ch.m[200], c.ch.s[200] = 3, 1
    c.ch.b[1400 + 700] = U.HIGH
    c.ch.m[1300], c.ch.s[1300] = 1, 0
    c.ch.m[1400 + 5], c.ch.s[1400 + 5] = U.LOW, 62
    acc = U.product(c.a, c.w) + c.ch.bias()
    c.acc = (acc + 2 ** 31) % 2 ** 32 - 2 ** 31
    run(c, "persistent gated, any constants")
    ran("gated_stream_kernel")
    c = U.Gated(9 + act, 700, 300, 256, act, bias=False)
    c.params.out_dy.m, c.params.out_dy.s = 1, 20
    run(c, "persistent gated, a small shift")
    if act:
        c.params.gelu.out.m, c.params.gelu.out.s = -3, 32
        run(c, "persistent gated, gelu's small shift")
        # a scale so fine that erf's table finds no room
        c = U.Gated(11, 700, 300, 256, act)
        c.params.gelu = B.ibert_gelu_params_from_scale(1 / 1500, 1 / 6000)
        assert c.params.gelu.q_b < -1700
        c.ch.m[:300] = c.ch.m[:300] // 8
        run(c, "persistent gated, gelu computed")
        ran("gated_stream_kernel<0")


@pytest.mark.parametrize("act", [0, 1], ids=["silu", "gelu"])
def test_persistent_gated_shifts_from_31_on(persistent, act):
    # one side of the fast epilogue's first shift and the other, multipliers at their ends, in the channels and behind the product
    for K, shift in ((128, 32), (256, 32), (144, 33), (128, 31)):
        c = U.Gated(K + act, 300, 140, K, act)
        c.ch.s[:] = shift
        c.ch.m[:] = c.ch.m // 8
        c.ch.m[[3, 150]], c.ch.m[[5, 153]] = 2 ** 31 - 1, U.LOW
        c.ch.b[[3, 5, 150]] = 2 ** 30 - 2 ** 23
        c.ch.b[[4, 153]] = 2 ** 23 - 2 ** 30
        acc = U.product(c.a, c.w) + c.ch.bias()
        assert abs(acc).max() < 2 ** 31
        c.acc = acc
        run(c, "persistent gated, K %d, shift %d" % (K, shift))
        c.params.out_dy.m, c.params.out_dy.s = (2 ** 31 - 1 if act else U.LOW), shift
        run(c, "persistent gated, K %d, shift %d behind the product" % (K, shift))
    ran("gated_stream_kernel")


@pytest.mark.parametrize("form", [(0, 0), (0, 1), (0, 3), (-1, -1)], ids=["tall", "low", "narrow", "rows"])
@pytest.mark.parametrize("K", [65520, 66560])
def test_gated_sums_at_the_end_of_32_bits(gpu, form, K):
    # codes of -128 throughout and a bias next to 2^30: sums of 2^31 - 2^18 and, past the end of INT32, beyond it, where they wrap in every kernel
    from paper_2101_01321_amd import binding as B
    M = 3 if form[0] < 0 else 33
    c = U.Gated(5, M, 20, K, 0)
    c.a[:], c.w[:] = -128, -128
    c.ch.b[:] = 2 ** 30 - 1
    c.ch.m[:], c.ch.s[:] = 2 ** 30, 47
    c.acc = (U.product(c.a, c.w) + c.ch.bias() + 2 ** 31) % 2 ** 32 - 2 ** 31
    assert bool((c.acc < 0).all()) == (K > 65536)
    B.ibert_rows_override(*form)
    try:
        run(c, "gated, K %d, %d rows" % (K, M))
        ran("rows_ring_kernel" if form[0] < 0 else "gated_stream_kernel")
    finally:
        B.ibert_rows_override(-1, -1)


@pytest.mark.parametrize("off", [0, 1, 4, 13])
@pytest.mark.parametrize("ld", [(0, 0, 0), (16, 32, 16), (3, 5, 7), (12, 4, 1)])
def test_rows_at_any_address(gpu, ld, off):
    for M, N, K in ((3, 37, 144), (20, 70, 256), (70, 50, 200)):
        run(U.Gated(M, M, N, K, M % 2, ld=ld), "i8 gated, strides %s, at %d" % (ld, off), off)
        run(U.Gated(M, M, N, K, M % 2, 64, True, ld=ld), "w4 gated, strides %s, at %d" % (ld, off), off)
        run(U.Rows4(M, M, N, K, 32, False, "i8", True, ld=ld), "w4, strides %s, at %d" % (ld, off), off)


@pytest.mark.parametrize("K", [4096, 4097, 20000, 1 << 17])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_sums_beyond_32_bits(gpu, group, zeros, K):
    # every product at its largest: 4096 of them just fit 32 bits, all of them take up to 37 and are cut off at INT32's end; the last row is small
    for M in (1, 20, 50):
        c = U.Rows4(K, M, 20, K, group, zeros, "i32", extreme=True)
        c.a[-1] = 1
        c.ch.m[:], c.ch.s[:] = 1 << 30, 30
        acc = U.product(c.a, c.w4.whole()) + c.ch.bias()
        assert acc.max() > U.HIGH or K <= 4097 or M == 1
        c.acc = np.clip(acc, U.LOW, U.HIGH)
        run(c, "w4 extreme, groups of %d, K %d" % (group, K))


def test_w4_ignores_what_stands_past_the_weights(gpu):
    torch, G, B = libs()
    c = U.Rows4(5, 6, 35, 150, 32, True, "i16")
    d = OnDevice(c)
    w, s, z = d.keep[0]
    real = U.W4.__new__(U.W4)
    real.w, real.s, real.z, real.group = np.full((35, 150), -1, np.int8), np.ones((35, 5), np.uint8), np.ones((35, 5), np.int8), 32
    rw, rs, rz = (G.to_dev(x) for x in real.pack())
    lo, hi = (rw & 15) == 0, (rw >> 4) == 0                         # nibbles that no weight has
    w |= torch.where(lo, 9, 0).to(torch.uint8) | torch.where(hi, 0x60, 0).to(torch.uint8)
    s[rs == 0] = 201
    z[rz == 0] = 5
    G.say("w4 with filled padding")
    d.call()
    torch.cuda.synchronize()
    d.check("w4 with filled padding")


@pytest.mark.parametrize("group", [None, 128])
def test_gated_without_biases(form, group):
    for M, F, K in ((3, 50, 256), (40, 33, 100)):
        run(U.Gated(M, M, F, K, M % 2, group, bias=False), "gated without biases, group %s" % group)


def test_constants_at_their_ends(gpu):
    # shifts of 0 and 62, multipliers of both signs and of INT32's ends, biases that push a sum to an end
    for group in (None, 64):
        c = U.Gated(9, 5, 24, 128, 0, group)
        for i, (m, s) in enumerate([(1, 0), (-1, 0), (U.HIGH, 62), (U.LOW, 62), (U.HIGH, 31), (U.LOW, 32), (0, 5), (U.LOW, 0)]):
            c.ch.m[i::8], c.ch.s[i::8] = m, s
        if group:
            c.ch.b[::5], c.ch.b[1::5] = U.HIGH, U.LOW
            acc = U.product(c.a, np.concatenate([c.g4.whole(), c.u4.whole()])) + c.ch.bias()
            c.acc = np.clip(acc, U.LOW, U.HIGH)
        run(c, "gated, ends, group %s" % group)
    c = U.Rows4(10, 7, 40, 256, 128, True, "i32", residual=True)
    c.ch.m[::3], c.ch.s[::3] = U.LOW, 62
    c.ch.m[1::3], c.ch.s[1::3] = U.HIGH, 0
    c.res_dy = (U.LOW, 0)
    run(c, "w4, ends")


def test_dtype_and_rows_that_are_not_there(gpu):
    torch, G, B = libs()
    c = U.Gated(3, 4, 20, 64, 0)
    d = OnDevice(c)
    before = d.out.clone()
    for change in ({"M": 0}, {"F": 0}):
        desc = c.desc()
        for k, v in change.items():
            setattr(desc, k, v)
        B.ibert_gemm_i8_gated(desc, d.a, d.w, d.b, d.m, d.s, d.out)
    torch.cuda.synchronize()
    assert torch.equal(before, d.out)


@pytest.mark.parametrize("kind", ["gated", "persistent", "w4_gated", "w4"])
def test_streams_and_graphs(gpu, kind):
    # two calls at once on streams of their own; then both captured, replayed between eager calls with other inputs
    torch, G, B = libs()
    make = {"gated": lambda i: U.Gated(i, 37, 200, 512, i % 2), "persistent": lambda i: U.Gated(i, 700, 1000, 256, i % 2), "w4_gated": lambda i: U.Gated(i, 3, 200, 512, i % 2, 64, True),
            "w4": lambda i: U.Rows4(i, 9, 300, 1024, 128, False, "i16", True)}[kind]
    d = [OnDevice(make(i)) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in d]
    torch.cuda.synchronize()
    G.say(kind + " on two streams")
    for _ in range(20):
        for x, s in zip(d, streams):
            x.call(s)
    torch.cuda.synchronize()
    for x in d:
        x.check(kind + " on two streams")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in d:
            x.call()
    for i in range(3):
        other = make(10 + i)
        other.ch, old = d[0].c.ch, d[0].c
        d[0].a.copy_(torch.from_numpy(other.a.reshape(-1)).to(d[0].a.device).view_as(d[0].a))
        for x in d:
            x.out[:-x.guard].fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        whole = old.w4.whole() if kind == "w4" else (np.concatenate([old.g4.whole(), old.u4.whole()]) if kind == "w4_gated" else old.w)
        old.a = other.a
        old.acc = np.clip(U.product(other.a, whole) + old.ch.bias(), U.LOW, U.HIGH)
        for x in d:
            x.check(kind + " replayed")


# ------------------------------------------------------------------------------------------- logits
class DeviceLogits:
    def __init__(self, c, off=0, in_place=False):
        torch, G, B = libs()
        self.c, dev = c, G.to_dev
        self.t = {k: dev(getattr(c, k)) for k in ("params", "tokens", "start", "made", "ids", "values", "bstart")}
        self.masks = dev(c.masks.view(np.int32)) if c.num_masks else None
        self.x = moved(dev(c.x), off)
        self.in_place = in_place
        self.y = self.x if in_place else moved(torch.cat([dev(c.y0).reshape(-1), torch.full((64,), 77, dtype=torch.int32, device=G.DEV)]), off)

    def call(self, stream=None):
        torch, G, B = libs()
        t, desc = self.t, self.c.desc()
        if self.in_place:
            desc.ldy = desc.ldx
        some = lambda k, n: t[k] if n else None      # noqa: E731
        B.ibert_logits_adjust_i(desc, self.x, t["params"], some("tokens", desc.num_tokens), some("start", desc.num_tokens), some("made", desc.num_tokens),
                                some("ids", desc.num_biases), some("values", desc.num_biases), some("bstart", desc.num_biases), self.masks, self.y, stream)

    def check(self, what):
        c = self.c
        if self.in_place:
            same(self.x, c.expected(c.x), what)
        else:
            same(self.y[:c.y0.size], c.expected(), what)
            assert bool((self.y[c.y0.size:] == 77).all()), "wrote past the end: " + what
            same(self.x, c.x, what + ", the input")


def _logits_cases():
    yield "one token", U.Logits(0, [3], 1, [1], 1)
    yield "seven tokens", U.Logits(1, [3, 0], 7, [3, 0], 2)
    yield "no history", U.Logits(2, [0, 0, 0], 333, None, 3)
    yield "plain", U.Logits(3, [0], 100)
    yield "biases alone", U.Logits(4, [0, 0], 500, [40, 3])
    yield "masks alone", U.Logits(5, [0] * 7, 1031, None, 4)
    for vocab in (31, 32, 33, 2047, 2048, 2049, 5003, 9000):
        yield "vocabulary of %d" % vocab, U.Logits(vocab, [0, 500, 77, 1, 3000], vocab, [9, 0, 300, 1, 2], vocab % 5)
    yield "a history longer than the vocabulary", U.Logits(6, [70000, 5], 300, [1000, 0], 2)
    yield "strides", U.Logits(7, [40, 50, 60], 2050, [4, 5, 6], 3, (3, 5, 2))
    yield "strides of four", U.Logits(8, [40, 50, 60], 2050, [4, 5, 6], 3, (2, 6, 0))


@pytest.mark.parametrize("name,case", list(_logits_cases()), ids=lambda v: v.replace(" ", "_") if isinstance(v, str) else "")
def test_logits(gpu, name, case):
    torch, G, B = libs()
    for off, in_place in ((0, False), (1, False), (0, True), (3, True)):
        G.say("logits: %s, at %d%s" % (name, off, ", in place" if in_place else ""))
        d = DeviceLogits(case, off, in_place)
        d.call()
        torch.cuda.synchronize()
        d.check(name)


def test_logits_clamp_what_the_device_says(gpu):
    # starts beyond the arrays and out of order, shifts outside [0, 62]: clamped, nothing is read outside
    torch, G, B = libs()
    c = U.Logits(11, [50, 60, 70, 80], 400, [20, 30, 10, 5], 2)
    c.start[:] = (-7, 10 ** 9, 100, U.LOW, U.HIGH)
    c.made[:] = (U.LOW, 10 ** 8, 120, 100)
    c.bstart[:] = (30, 20, -1, 10 ** 9, 40)
    c.params[0, 1], c.params[1, 3], c.params[2, 1], c.params[3, 1] = 63, -1, U.HIGH, U.LOW
    d = DeviceLogits(c)
    G.say("logits: values that are clamped")
    d.call()
    torch.cuda.synchronize()
    d.check("clamped")


def test_logits_streams_and_graphs(gpu):
    torch, G, B = libs()
    d = [DeviceLogits(U.Logits(20 + i, [300, 5, 60], 3001, [7, 0, 9], 3)) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in d]
    torch.cuda.synchronize()
    G.say("logits on two streams")
    for _ in range(20):
        for x, s in zip(d, streams):
            x.call(s)
    torch.cuda.synchronize()
    for x in d:
        x.check("two streams")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in d:
            x.call()
    for i in range(3):
        c = d[0].c
        other = U.Logits(30 + i, [300, 5, 60], 3001, [7, 0, 9], 3)
        c.tokens[:], c.made[:] = other.tokens, other.made
        d[0].t["tokens"].copy_(torch.from_numpy(c.tokens))
        d[0].t["made"].copy_(torch.from_numpy(c.made))
        for x in d:
            x.y[:x.c.y0.size].fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        for x in d:
            x.check("replayed")


def test_more_rows_than_a_launch_holds(gpu):
    # 2^19 blocks of 32 rows of one channel tile, 2^22 rows of one slice: a second launch takes what is left
    torch, G, B = libs()
    M = (1 << 19) * 32 + 5
    G.say("w4, %d rows" % M)
    a = torch.randint(-128, 128, (M,), device=G.DEV, dtype=torch.int8)
    w, s, _ = B.ibert_w4_pack(np.array([[-3]], np.int8), np.array([[5]], np.uint8), None, 32)
    w, s, one = G.to_dev(w), G.to_dev(s), torch.ones(1, dtype=torch.int32, device=G.DEV)
    out = torch.zeros(M + 9, dtype=torch.int16, device=G.DEV)
    B.ibert_gemm_w4_requant(B.W4Desc(M, 1, 1, B.I16, 1, 1, 0, 32767, B.Dyadic(1, 0)), a, B.W4Weights(w.data_ptr(), s.data_ptr(), None, 32), None, one, one * 0, None, out)
    torch.cuda.synchronize()
    assert torch.equal(out[:M], a.to(torch.int16) * -15) and not out[M:].any()
    M = 2 ** 31 - 1
    G.say("w4 and a gated block, %d rows" % M)
    a = torch.randint(-8, 9, (M,), device=G.DEV, dtype=torch.int8)
    out = torch.zeros(M, dtype=torch.int8, device=G.DEV)
    B.ibert_gemm_w4_requant(B.W4Desc(M, 1, 1, B.I8, 1, 1, 0, 127, B.Dyadic(1, 0)), a, B.W4Weights(w.data_ptr(), s.data_ptr(), None, 32), None, one, one * 0, None, out)
    torch.cuda.synchronize()
    for x, y in zip(a.split(1 << 28), out.split(1 << 28)):
        assert torch.equal(y, (x.to(torch.int16) * -15).clamp(-127, 127).to(torch.int8))
    p = B.ibert_gate_params_from_scales(B.GATE_SILU, 0, 1 / 32767, 1.0)
    p.out_dy = B.Dyadic(1, 20)
    m, sh = torch.tensor([1 << 12, 1 << 10], dtype=torch.int32, device=G.DEV), torch.zeros(2, dtype=torch.int32, device=G.DEV)
    B.ibert_gemm_i8_gated(B.GatedDesc(M, 1, 1, 1, 1, 1, p), a, torch.ones(2, dtype=torch.int8, device=G.DEV), None, m, sh, out)
    torch.cuda.synchronize()
    v = np.arange(-8, 9)
    want = torch.from_numpy(U.gate(v[:, None] * 1, v[:, None] * 1, m.cpu().numpy(), sh.cpu().numpy(), p)[:, 0]).to(G.DEV)
    assert want.unique().numel() == 7        # (of gates of -2.8 and less this output scale leaves nothing)
    for x, y in zip(a.split(1 << 27), out.split(1 << 27)):
        assert torch.equal(y, want[x.to(torch.int32) + 8])
    del a, out
    rows = (1 << 22) + 3
    G.say("logits, %d rows" % rows)
    x = torch.randint(-9, 9, (rows,), device=G.DEV, dtype=torch.int32)
    x[-1] = U.LOW
    params = torch.tensor([1, 0, 1, 0, 5, 7, -1], dtype=torch.int32, device=G.DEV).repeat(rows, 1)
    made = torch.zeros(rows + 1, dtype=torch.int32, device=G.DEV)
    made[rows - 1:] = torch.tensor([0, 2], device=G.DEV)      # the last but one row's two tokens are its own
    y = torch.full((rows + 9,), 77, dtype=torch.int32, device=G.DEV)
    start = made.clone()
    start[rows - 1], start[rows] = 2, 2                       # row rows - 2 has tokens [0, 2)
    B.ibert_logits_adjust_i(B.LogitsDesc(rows, 1, 1, 1, 2, 0, 0, 0), x, params, torch.zeros(2, dtype=torch.int32, device=G.DEV), start, made, None, None, None, None, y)
    torch.cuda.synchronize()
    want = x.clone()
    want[rows - 2] -= 5 + 2 * 7
    assert torch.equal(y[:rows], want) and bool((y[rows:] == 77).all())


# ------------------------------------------------------------------------------------------- the run of them
@pytest.mark.parametrize("M,group", [(1, 32), (5, 128), (70, 64)])
def test_a_decoder_s_feed_forward_and_head(gpu, M, group):
    """LayerNorm -> gated block (INT8 and 4-bit weights) -> down projection + residual -> LayerNorm -> head -> penalties -> Softmax, each step against its
    definition on what the step before left."""
    import oracle
    torch, G, B = libs()
    H, F, V = 256, 344, 700
    rng = np.random.default_rng(M)
    gq, bq, sh = B.ibert_layernorm_params_from_float(rng.normal(1, 0.1, H), rng.normal(0, 0.1, H), 1 / 32)
    tg, tb = G.to_dev(gq), G.to_dev(bq)
    x = G.to_dev(rng.integers(-9000, 9000, (M, H)).astype(np.int16))
    h = torch.zeros(M, H, dtype=torch.int8, device=G.DEV)
    G.say("feed-forward and head of %d tokens" % M)
    for w4 in (False, True):
        B.ibert_layernorm_i16(x, h, M, H, H, H, tg, tb, sh)
        g = U.Gated(M, M, F, H, int(w4), group if w4 else None)
        dg = OnDevice(g)
        dg.a = h
        dg.call()
        c = U.Rows4(M + 1, M, H, F, group, True, "i16", residual=True)
        dc = OnDevice(c)
        dc.a, dc.r = dg.out, h
        dc.call()
        y = torch.zeros(M, H, dtype=torch.int8, device=G.DEV)
        B.ibert_layernorm_i16(dc.out, y, M, H, H, H, tg, tb, sh)
        head = U.Rows4(M + 2, M, V, H, group, False, "i32")
        m, s = U.dyadic(400 / (40 * 150 * 3 * 16.0))
        head.ch.m[:], head.ch.s[:] = m, s
        dh = OnDevice(head)
        dh.a = y
        dh.call()
        lg = U.Logits(M, [20] * M, V, [3] * M, 2)
        lg.params[:, 6] = np.where(np.arange(M) % 2, -1, 0)
        lg.params[:, :4] = (*U.dyadic(1 / 1.2), *U.dyadic(1.2))
        lg.values[:] = np.clip(lg.values, -500, 500)
        lg.params[:, 4:6] = (50, 7)
        dl = DeviceLogits(lg)
        dl.x = dh.out
        dl.call()
        probs = torch.zeros(M, V, dtype=torch.int32, device=G.DEV)
        sp = B.ibert_softmax_params_from_scale(np.log(2) / 64, V, 20, B.I32)
        B.ibert_softmax_i(dl.y, probs, M, V, V, V, sp)
        torch.cuda.synchronize()
        # the same, step by step
        hn = h.cpu().numpy()
        g.acc = np.clip(U.product(hn, np.concatenate([g.g4.whole(), g.u4.whole()]) if w4 else g.w) + g.ch.bias(), U.LOW, U.HIGH)
        dg.check("gated")
        c.a, c.r = dg.out[:M * F].cpu().numpy().reshape(M, F), hn
        c.acc = np.clip(U.product(c.a, c.w4.whole()) + c.ch.bias(), U.LOW, U.HIGH)
        dc.check("down projection")
        yn = y.cpu().numpy()
        same(y, oracle.layernorm(c.expected().astype(np.int32), gq, bq, sh), "layernorm")
        head.acc = np.clip(U.product(yn, head.w4.whole()) + head.ch.bias(), U.LOW, U.HIGH)
        dh.check("head")
        lg.x = head.expected()
        want = lg.expected()
        same(dl.y[:want.size], want, "logits")
        z = want.astype(np.int64).max(1, keepdims=True) - want
        q_ln2, q_b, q_c = sp.q_ln2, sp.q_b, sp.q_c
        z, rest = z // q_ln2, z % q_ln2
        e = np.where(z < 31, ((q_b - rest) ** 2 + q_c) >> np.minimum(z, 31), 0)
        p = (e * (2 ** 31 // e.sum(1, keepdims=True)) + (1 << 10 >> 0)) >> 11
        same(probs, p, "softmax")
        masked = want == U.LOW
        assert masked[::2].any() and not probs.cpu().numpy()[masked].any()
