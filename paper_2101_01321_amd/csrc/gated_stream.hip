// The gated block for many tokens: the persistent workgroups of gemm_stream.h (streamed K steps of 128 bytes, two LDS stages, a step in
// four phases by quadrants of the wavefront's tile), whose tile is 256 or 128 tokens by 128 channels of the gate and the same 128 of the up
// projection, or 128 tokens by 64 of each, by four wavefronts.
//
//   * The first two MFMA blocks of a wavefront's four are rows of W_gate and the last two the same rows of W_up, so that the two halves of
//     a step ("W first", "W second") bring one matrix each, and a lane ends up with gate and up sums of the same two neighbouring channels
//     in registers: neither product is ever stored.
//   * Rows of W are dealt to the LDS rows such that lane r of 16 has channels 2 r and 2 r + 1 of its wavefront's 32.
//   * F and M may be ragged: operands, constants and output are buffers that end with the last row or channel.
//   * SiLU's sigmoids, and GELU's erf where it has room, are tables in LDS, built once by every workgroup with the function they stand for.
//
// What bounds it: where K is long the matrix units at the clock that power leaves (8192 x 4096 -> 2 x 12288 636 to 671 us by the card, 2.6 to 2.5 POP/s, MFMA busy 0.72); where it is short the
// epilogue, 20 ALU instructions a value that no MFMA runs beside (2741 x 1024 -> 2 x 4096 31 to 34 us: a tile of 128 x 128 takes 4.7 us in its loop and 3.5 in its
// epilogue), and the last round of tiles, three quarters full there.  Three tiles: 256 tokens read W half as often; 128 fill more units; 128 x 64, two workgroups to a unit,
// fill them where 128 x 128 tiles do not (256 x 1024 -> 2 x 4096 11.9 / 9.3 us; see plan_gated).  Where both of a unit's workgroups have work they gain nothing of each
// other's epilogues, with wave priorities that would put them out of phase neither (2741 tokens: 33.8 us with any).
#include "gate_math.h"
#include "gemm_stream.h"
#include "gated_stream.h"

namespace ibert {

struct GatedStreamArgs {
    const int8_t* A;
    const int8_t* W;
    const int32_t* bias;
    const int32_t* mult;
    const int32_t* shift;
    int8_t* C;
    int32_t M, F, K, nk;           // nk: steps of 128 bytes in K
    int32_t lda, ldw, ldc;
    int32_t tiles_m, bn;           // as in StreamArgs
    uint32_t bn_magic;
    int32_t xs, gs, per_xcd;
    int32_t fast;                  // K * 128^2 < 2^30, the product's shift in [32, 62], and gelu_fast_ok where it is GELU
    int32_t c_vec;                 // rows of C allow 16-byte stores
    GateConst gate;
};

constexpr int GS_PITCH = 48, GS_TURN_WAVE = 32 * GS_PITCH;
// BM: tokens of a tile; BF: its channels (of each matrix).
template <int BM, int BF>
struct GatedLayout {
    static constexpr int NW = BF / 16, UNIT = 128 / BF;  // wavefronts; workgroups that a compute unit holds
    static constexpr int STAGE = (BM + 2 * BF) * 128;
    static constexpr int PAR = 2 * STAGE;                // two buffers of 3 x 2 BF constants
    static constexpr int TURN = PAR + 2 * 3 * 2 * BF * 4;   // rows on their way out: 32 rows of 32 bytes a wavefront
    static constexpr int TABLE = TURN + NW * GS_TURN_WAVE;
    static constexpr int ERF = BF == 128 ? 3400 : 1792;     // entries that GELU's table may have
    static constexpr int LDS = TABLE + 4 * ERF;
    static_assert(LDS <= 163840 / UNIT && 2 * (2 * SIG_STEPS + 1) <= 4 * ERF, "LDS of a unit's workgroups");
};

enum { GS_GELU = 0, GS_SILU = 1, GS_GELU_TABLE = 2 };

// TAIL: K is no multiple of 128 (of 16 it is).
template <int ACT, int BM, int BF, bool TAIL>
__global__ __launch_bounds__(4 * BF, 2) void gated_stream_kernel(GatedStreamArgs g)
{
    using GL = GatedLayout<BM, BF>;
    constexpr int GS_STAGE = GL::STAGE, GS_PAR = GL::PAR, BN = 2 * BF, NW = GL::NW, NT = 64 * NW, WR = 2, WC = NW / 2;
    constexpr int WM = BM / WR, WN = BN / WC, FM = WM / 16, FN = 4, FMH = FM / 2, FN0 = 2, FN1 = 2;
    constexpr int QA = FMH * 2 * WR / NW, QW = FN0 * 2 * WC / NW, NQ = QA + QW;       // requests of a wavefront: A half, W half, a group
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = wave % WR * WM, wn0 = wave / WR * WN;
    const int frow = lane & 15, fch = lane >> 4;

    // ---- the workgroup's tiles (see stream_run, stream_tile) ------------------------------------
    const int xcd = blockIdx.x & 7, group = g.tiles_m * g.bn, xm = xcd >> g.xs, t0 = (int)(((int64_t)xm * group) >> g.gs);
    const int first_col = (xcd & ((1 << g.xs) - 1)) * g.bn, count = (int)(((int64_t)(xm + 1) * group) >> g.gs) - t0;
    const uint32_t kbytes = (uint32_t)g.nk * 128u;
    int lt = blockIdx.x >> 3;
    if (lt >= count) return;
    auto tile_at = [&](int l, int& m0, int& n0) {
        const int t = t0 + l, tm = udiv_fix(t, g.bn, g.bn_magic);
        m0 = tm * BM;
        n0 = (first_col + t - tm * g.bn) * BF;
    };

    // ---- requests (see gemm_stream.h) -----------------------------------------------------------
    const int r8 = lane >> 3;
    const uint32_t chunk = (uint32_t)(((lane & 7) ^ (((wave & 1) << 2) | (r8 >> 1))) << 4);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t*)lds;
    auto first_row = [&](int nb, int rows) { return wave / nb * rows + wave % nb * 8; };
    constexpr int SA = NW / (FMH * 2) * WM, SW = NW / (FN0 * 2) * WN;                // rows of the stage from request to request
    const int pa = first_row(FMH * 2, WM), pw = first_row(FN0 * 2, WN);              // (the up projection's: 32 rows of the stage on)
    auto w_row = [&](int p) {                                      // channel, from the tile's first, that belongs in row p of the stage's W part
        const int w = p / WN, r = p - w * WN, q = (r & 8) + r8;
        return w * 32 + 2 * q + ((r >> 4) & 1);
    };
    uint32_t va[2][QA], vw[QW];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < QA; ++q) va[h][q] = (uint32_t)(pa + h * (WM / 2) + q * SA + r8) * (uint32_t)g.lda + chunk;
#pragma unroll
    for (int q = 0; q < QW; ++q) vw[q] = (uint32_t)w_row(pw + q * SW) * (uint32_t)g.ldw + chunk;
    v4i da, dg, du;                                                // descriptors of the request stream's tile: A, gate, up
    da[3] = dg[3] = du[3] = 0x00020000;
    uint32_t koff = 0, kinc = 128, rstage = lds0;
    int rlt = lt;
    auto buffer = [](v4i& d, const void* p, uint32_t bytes) {
        const uint64_t u = (uint64_t)(uintptr_t)p;
        d[0] = (int32_t)(uint32_t)u;
        d[1] = (int32_t)((uint32_t)(u >> 32) & 0xffffu);
        d[2] = (int32_t)bytes;
    };
    auto request_tile = [&](int l) {
        if (l < count) {
            int m0, n0;
            tile_at(l, m0, n0);
            const int rows = g.M - m0 < BM ? g.M - m0 : BM, cols = g.F - n0 < BF ? g.F - n0 : BF;
            buffer(da, g.A + (int64_t)m0 * g.lda, (uint32_t)(rows - 1) * (uint32_t)g.lda + (uint32_t)g.K);
            buffer(dg, g.W + (int64_t)n0 * g.ldw, (uint32_t)(cols - 1) * (uint32_t)g.ldw + (uint32_t)g.K);
            buffer(du, g.W + ((int64_t)g.F + n0) * g.ldw, (uint32_t)(cols - 1) * (uint32_t)g.ldw + (uint32_t)g.K);
            kinc = 128;
        } else {
            da[2] = dg[2] = du[2] = 0;
            kinc = 0;
        }
    };
    // In the last step of a TAIL the lanes whose bytes lie past K ask for A's outside its buffer: zeros, whatever they meet of W.
    uint32_t past = 0;
    auto mark_tail = [&]() {
        if constexpr (TAIL) past = koff + chunk >= (uint32_t)g.K ? 1u << 30 : 0u;
    };
    mark_tail();
    auto request_one = [&](int h, int q) {
        const bool is_a = q < QA;
        const int k = is_a ? q : q - QA;
        const int row = is_a ? h * (WM / 2) + k * SA : h * 32 + k * SW;
        const uint32_t place = rstage + (uint32_t)((is_a ? pa : BM + pw) * 128);
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds"
                     :: "s"(place), "i"(row * 128), "v"(is_a ? (TAIL ? va[h][is_a ? k : 0] + past : va[h][is_a ? k : 0]) : vw[is_a ? 0 : k]), "s"(is_a ? da : (h == 0 ? dg : du)), "s"(koff)
                     : "memory", "m0", "scc");
    };
    auto request_advance = [&]() {
        koff += kinc;
        rstage = 2 * lds0 + (uint32_t)GS_STAGE - rstage;
        if (koff == kbytes) {
            koff = 0;
            rlt += g.per_xcd;
            request_tile(rlt);
        }
        mark_tail();
    };
    // Constants of a tile: [bias, mult, shift][gate, up][BF], by DMA, 64 dwords a request; zeros past the last channel.
    int par_n0 = -1, par_buf = 1;
    auto request_constants = [&](int n0) {
        if (n0 == par_n0) return;
        par_n0 = n0;
        par_buf ^= 1;
        const uint32_t base = lds0 + (uint32_t)(GS_PAR + par_buf * 3 * BN * 4);
#pragma unroll
        for (int a = 0; a < 3; ++a) {
            const int32_t* src = a == 0 ? g.bias : (a == 1 ? g.mult : g.shift);
            if (src) {
#pragma unroll
                for (int c = 0; c < BN / 64; ++c)
                    if ((a * (BN / 64) + c) % NW == wave) {
                        v4i d;
                        buffer(d, src + (int64_t)(c * 64 / BF) * g.F, (uint32_t)g.F * 4u);
                        d[3] = 0x00020000;
                        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                                     :: "s"(base + (uint32_t)((a * BN + c * 64) * 4)), "v"((uint32_t)(n0 + c * 64 % BF + lane) * 4u), "s"(d) : "memory", "m0");
                    }
            } else {
                int32_t* p = reinterpret_cast<int32_t*>(lds + GS_PAR + par_buf * 3 * BN * 4) + a * BN;
                int32_t fill = 0, c0 = tid;
                asm volatile("" : "+s"(fill), "+v"(c0));
                for (int c = c0; c < BN; c += NT) p[c] = fill;
            }
        }
    };
    constexpr auto vm = [](int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); };

    v4i acc[FN][FM];
    const int rd0 = frow * 128 + ((fch ^ ((frow >> 1) & 7)) << 4);
    auto operand = [&](int sl, int off) { return *reinterpret_cast<const v4i*>(lds + off + (sl ? rd0 ^ 64 : rd0)); };
    v4i at[FMH][2], ab[FMH][2], w0[FN0][2], w1[FN1][2];
    int stage = 0;
    auto read_a = [&](v4i (&d)[FMH][2], int st, int h, int q) { d[q >> 1][q & 1] = operand(q & 1, st + (wm0 + (h * FMH + (q >> 1)) * 16) * 128); };
    auto read_w0 = [&](int st, int q) { w0[q >> 1][q & 1] = operand(q & 1, st + BM * 128 + (wn0 + (q >> 1) * 16) * 128); };
    auto read_w1 = [&](int st, int q) { w1[q >> 1][q & 1] = operand(q & 1, st + BM * 128 + (wn0 + (FN0 + (q >> 1)) * 16) * 128); };

    // ---- prologue -------------------------------------------------------------------------------
    int m0, n0;
    tile_at(lt, m0, n0);
    request_constants(n0);
    request_tile(lt);
    auto request_two_steps = [&]() {
#pragma unroll 1
        for (int st = 0; st < 2; ++st) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) request_one(0, q);
#pragma unroll
            for (int q = 0; q < NQ; ++q) request_one(1, q);
            request_advance();
        }
    };
    request_two_steps();
    // SiLU: the factor of a gate in step i - 1024 of either sign, 15 bits.  GELU: erf + q_1 of Alg. 2 over [q_b, -q_b], outside of which it stays the same.
    if constexpr (ACT == GS_SILU) {
        uint16_t* const sig = reinterpret_cast<uint16_t*>(lds + GL::TABLE);
        for (int d = tid; d <= 2 * SIG_STEPS; d += NT) {
            const int i = d - SIG_STEPS;
            const uint32_t p = sigmoid15((uint32_t)(i < 0 ? -i : i));
            sig[d] = (uint16_t)(i < 0 ? 32768u - p : p);
        }
    } else if constexpr (ACT == GS_GELU_TABLE) {
        int32_t* const erf = reinterpret_cast<int32_t*>(lds + GL::TABLE);
        for (int d = tid; d <= -2 * g.gate.gelu.q_b; d += NT) {
            const int q = d + g.gate.gelu.q_b, v = (q < 0 ? -q : q) + g.gate.gelu.q_b, poly = smad24(v, v, g.gate.gelu.q_c);
            erf[d] = (q < 0 ? -poly : (q == 0 ? 0 : poly)) + g.gate.gelu.q_1;
        }
    }
    __builtin_amdgcn_s_waitcnt(vm(2 * NQ));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

    auto quadrant = [&](v4i (&xw)[2][2], int i0, v4i (&xa)[FMH][2], int j0, auto zero_tag, auto&& between) {
        constexpr bool ZERO = decltype(zero_tag)::value;
#pragma unroll
        for (int sl = 0; sl < 2; ++sl)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < FMH; ++j) {
                    between((sl * 2 + i) * FMH + j);
                    __builtin_amdgcn_sched_barrier(0);
                    acc[i0 + i][j0 + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(xa[j][sl], xw[i][sl], ZERO && sl == 0 ? v4i{0, 0, 0, 0} : acc[i0 + i][j0 + j], 0, 0, 0);
                }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int MQ = 4 * FMH;                                    // MFMAs of a quadrant
    // One K step; REQ and wait as in gemm_stream.h.
    auto step = [&](auto req_tag, bool wait) {
        constexpr int REQ = decltype(req_tag)::value;
        using Z = std::integral_constant<bool, REQ == 2>;
        const int nst = GS_STAGE - stage;
        auto ask = [&](int h, int n, int idx) {
#pragma unroll
            for (int r = 0; r < 2 * NQ; ++r)
                if (r < n && idx == (2 * r + 1) * (2 * MQ) / (2 * n)) request_one(REQ == 2 ? (r < NQ ? 0 : 1) : h, REQ == 2 && r >= NQ ? r - NQ : r);
        };
        quadrant(w0, 0, at, 0, Z{}, [&](int idx) {
            if (idx < 2 * FN1) read_w1(stage, idx);
            if (REQ == 1) ask(0, NQ, idx);
        });
        quadrant(w1, FN0, at, 0, Z{}, [&](int idx) {
            if (idx < 2 * FMH) read_a(ab, stage, 1, idx);
            if (REQ == 1) ask(0, NQ, MQ + idx);
        });
        if (wait) __builtin_amdgcn_s_waitcnt(vm(REQ == 1 ? 2 * NQ : NQ));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        quadrant(w0, 0, ab, FMH, Z{}, [&](int idx) {
            if (idx < 2 * FMH) read_a(at, nst, 0, idx);
            ask(1, REQ == 2 ? 2 * NQ : NQ, idx);
        });
        quadrant(w1, FN0, ab, FMH, Z{}, [&](int idx) {
            if (idx < 2 * FN0) read_w0(nst, idx);
            ask(1, REQ == 2 ? 2 * NQ : NQ, MQ + idx);
        });
        request_advance();
        if (wait) __builtin_amdgcn_s_waitcnt(vm(2 * NQ));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        stage = nst;
    };

    bool first = true;
    using R1 = std::integral_constant<int, 1>;
    using R2 = std::integral_constant<int, 2>;
    for (;;) {
#pragma unroll
        for (int q = 0; q < 2 * FMH; ++q) read_a(at, stage, 0, q);
#pragma unroll
        for (int q = 0; q < 2 * FN0; ++q) read_w0(stage, q);
        step(R2{}, first);
        const int par_own = par_buf;
        if (lt + g.per_xcd < count) {
            int next_m0, next_n0;
            tile_at(lt + g.per_xcd, next_m0, next_n0);
            request_constants(next_n0);
        }
        for (uint32_t kt = 128; kt < kbytes; kt += 128) step(R1{}, true);

        // ---- epilogue ---------------------------------------------------------------------------
        // acc[i][j][e] (i < 2 gate, else up) = channel n0 + wn0 / 2 + 2 r16 + i % 2 of row m0 + wm0 + 16 j + 4 u + e
        int el = lane;
        asm volatile("" : "+v"(el));
        const int r16 = el & 15, u = el >> 4, wf0 = wn0 / 2;
        const int32_t* par = reinterpret_cast<const int32_t*>(lds + GS_PAR + par_own * 3 * BN * 4);
        typedef const __attribute__((address_space(4))) GatedStreamArgs* kernel_args;
#if defined(__HIP_DEVICE_COMPILE__)
        kernel_args ga = (kernel_args)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(ga));
#else
        kernel_args ga = nullptr;
#endif
        const int last = ga->M - 1 - m0, rows = last < BM ? last : BM - 1;
        const int cols = ga->F - n0 < BF ? ga->F - n0 : BF;
        const int64_t out0 = (int64_t)m0 * ga->ldc + n0;
        // Fast form: every shift of the tile's channels in [32, 62] (a multiplier below 1/2), every |bias| below 2^30, and `fast`.
        bool fast;
        {
            bool ok = true;
#pragma unroll
            for (int c = 0; c < BN; c += 64) {
                const int32_t ps = par[2 * BN + c + el], pb = par[c + el];
                if (c % BF + el < cols) ok = ok && ps >= 32 && ps <= 62 && (pb ^ (pb << 1)) >= 0;
            }
            fast = __builtin_amdgcn_ballot_w64(!ok) == 0 && ga->fast;
        }
        if (fast) {
            const auto cb = __builtin_amdgcn_make_buffer_rsrc(ga->C + out0, 0, (int)((uint32_t)rows * (uint32_t)ga->ldc + (uint32_t)cols), 0x00020000);
            int64_t c0[FN];
            int32_t mm[FN], sh[FN];
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const int c = (i >> 1) * BF + wf0 + 2 * r16 + (i & 1);
                const int32_t b = par[c], s = par[2 * BN + c];
                mm[i] = par[BN + c];
                c0[i] = (int64_t)b * mm[i] + ((int64_t)1 << ((s - 1) & 63));
                sh[i] = (s - 32) & 31;
            }
            const GeluConst gl{ga->gate.gelu.q_b, ga->gate.gelu.q_c, ga->gate.gelu.q_1, ga->gate.gelu.q_max, ga->gate.gelu.m, ga->gate.gelu.s};
            // (x m + 2^(s-1)) >> s of a 32-bit x, s in [32, 62]: the high half of one 64-bit multiply-add, shifted; below 2^30 + 1 in size
            const int64_t gl_rnd = (int64_t)1 << ((gl.s - 1) & 63), ornd = (int64_t)1 << ((ga->gate.s - 1) & 63);
            const int32_t gl_sh = (gl.s - 32) & 31, om = ga->gate.m, osh = (ga->gate.s - 32) & 31;
            const uint32_t table = lds0 + (uint32_t)GL::TABLE;
            int8_t* const turn = lds + GL::TURN + wave * GS_TURN_WAVE;
            auto value = [&](int i, int n) { return (int32_t)(((int64_t)acc[i][n >> 2][n & 3] * mm[i] + c0[i]) >> 32) >> sh[i]; };
            auto fence = []() { __builtin_amdgcn_wave_barrier(); };
            typedef unsigned v4u __attribute__((ext_vector_type(4)));
            typedef const __attribute__((address_space(3))) uint16_t* lds_halves;
            typedef const __attribute__((address_space(3))) int32_t* lds_words;
            constexpr int UNITS = FM / 2;
            v4u mv[UNITS];
            const int col = wf0 + (el & 1) * 16, mrow = el >> 1;   // piece and row of a unit that the lane moves
            auto store = [&](int unit) __attribute__((always_inline)) {
                const int row = wm0 + unit * 32 + mrow, at = row * ga->ldc + col;
                if (ga->c_vec && col + 16 <= cols) __builtin_amdgcn_raw_buffer_store_b128(mv[unit], cb, at, 0, 0);
                else if (row <= last) {
                    int8_t* const p = ga->C + out0 + at;
                    if (col + 16 <= cols) __builtin_memcpy(p, &mv[unit], 16);
                    else {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (col + e < cols) p[e] = (int8_t)(mv[unit][e >> 2] >> (8 * (e & 3)));
                    }
                }
            };
            // the results of token n: table reads of both channels first
            auto results = [&](int n) __attribute__((always_inline)) {
                int32_t gt[2], f[2], up[2], y[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (ACT == GS_SILU) {
                        gt[i] = med3_const<-65535, 65535>(value(i, n));
                        // (|g| + 8) >> 4 with g's sign: below zero the shift rounds the other way
                        const int32_t d = med3_const<-SIG_STEPS, SIG_STEPS>((gt[i] + 8 + (gt[i] >> 31)) >> 4);
                        f[i] = *(lds_halves)(uintptr_t)(table + 2 * SIG_STEPS + (uint32_t)(d << 1));
                    } else {
                        gt[i] = med3_i32(value(i, n), -gl.q_max, gl.q_max);
                        if constexpr (ACT == GS_GELU_TABLE) f[i] = *(lds_words)(uintptr_t)(table + (uint32_t)((med3_i32(gt[i], gl.q_b, -gl.q_b) - gl.q_b) << 2));
                        else {
                            const int32_t v = min(max(gt[i], -gt[i]), -gl.q_b) + gl.q_b;
                            const int32_t poly = smad24(v, v, gl.q_c), sg = gt[i] >> 31;
                            f[i] = ((poly ^ sg) - sg) + gl.q_1;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) up[i] = med3_i32(value(2 + i, n), -32767, 32767);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    int32_t a;
                    if constexpr (ACT == GS_SILU) a = smad24(gt[i], f[i], 16384) >> 15;
                    else a = med3_const<-32767, 32767>((int32_t)(((int64_t)smul24(gt[i], f[i]) * gl.m + gl_rnd) >> 32) >> gl_sh);
                    y[i] = med3_const<-127, 127>((int32_t)(((int64_t)smul24(a, up[i]) * om + ornd) >> 32) >> osh);
                }
                return (uint16_t)__builtin_amdgcn_perm((uint32_t)y[1], (uint32_t)y[0], 0x0c0c0400u);
            };
#pragma unroll
            for (int unit = 0; unit < UNITS; ++unit) {
                fence();
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    *reinterpret_cast<uint16_t*>(turn + (16 * (t / 4) + 4 * u + t % 4) * GS_PITCH + 2 * r16) = results(8 * unit + t);
                    if (t % 2 == 1) __builtin_amdgcn_sched_barrier(0);
                }
                fence();
                mv[unit] = *reinterpret_cast<const v4u*>(turn + mrow * GS_PITCH + (el & 1) * 16);
                // before the first store this wavefront's requests have all landed, so that the next tile's first step need not count stores among loads
                if (unit == 1) __builtin_amdgcn_s_waitcnt(vm(0));
                if (unit >= 1) store(unit - 1);
            }
            store(UNITS - 1);
        } else {
            // Any constants: a rolled loop, 16 rows of each row of wavefronts at a time through LDS, where the next tile's first steps had
            // arrived -- they are requested again afterwards.
            constexpr int SP = BN + 4;
            int32_t* const st = reinterpret_cast<int32_t*>(lds);
            __builtin_amdgcn_s_waitcnt(vm(0));
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll 1
            for (int j = 0; j < FM; ++j) {
#pragma unroll
                for (int k = 0; k < FM; ++k)
                    if (k == j) {
#pragma unroll
                        for (int i = 0; i < FN; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) st[(wave % WR * 16 + 4 * u + e) * SP + (i >> 1) * BF + wf0 + 2 * r16 + (i & 1)] = acc[i][k][e];
                    }
                __syncthreads();
#pragma unroll 1
                for (int q = wave * 64 + el; q < 16 * WR * BF; q += NT) {
                    const int r = q / BF, c = q - r * BF, row = (r >> 4) * WM + 16 * j + (r & 15);
                    if (row > last || c >= cols) continue;
                    const GateConst gc{ga->gate.silu, GeluConst{ga->gate.gelu.q_b, ga->gate.gelu.q_c, ga->gate.gelu.q_1, ga->gate.gelu.q_max, ga->gate.gelu.m, ga->gate.gelu.s},
                                       ga->gate.m, ga->gate.s};
                    ga->C[out0 + (int64_t)row * ga->ldc + c] =
                        (int8_t)gate_one((int32_t)((uint32_t)st[r * SP + c] + (uint32_t)par[c]), (int32_t)((uint32_t)st[r * SP + BF + c] + (uint32_t)par[BF + c]),
                                         par[BN + c], par[2 * BN + c] & 63, par[BN + BF + c], par[2 * BN + BF + c] & 63, gc);
                }
                __syncthreads();
            }
            rlt = lt + g.per_xcd;
            koff = 0;
            rstage = lds0 + (uint32_t)stage;
            request_tile(rlt);
            mark_tail();
            request_two_steps();
            __builtin_amdgcn_s_waitcnt(vm(0));
            asm volatile("s_barrier" ::: "memory");
        }
        lt += g.per_xcd;
        if (lt >= count) break;
        tile_at(lt, m0, n0);
        first = false;
    }
}

bool gated_stream_ok(const ibert_gated_desc& d, const int8_t* A, const int8_t* W)
{
    return d.K % 16 == 0 && aligned(A, 16) && aligned(W, 16) && d.lda % 16 == 0 && d.ldw % 16 == 0 && d.lda < (1 << 20) && d.ldw < (1 << 20) && d.ldc < (1 << 20) &&
           (((int64_t)d.M + 127) / 128) * ((d.F + 63) / 64) < (1 << 26);
}

template <int ACT, int BM, int BF, bool TAIL>
static int launch_gated_stream_as(GatedStreamArgs& s, int64_t weight_bytes, hipStream_t stream)
{
    s.tiles_m = (int32_t)(((int64_t)s.M + BM - 1) / BM);
    using GL = GatedLayout<BM, BF>;
    const int tiles_n = (s.F + BF - 1) / BF;
    // as stream_shares and stream_deal
    s.xs = 0;
    while (s.xs < 2 && tiles_n % (2 << s.xs) == 0 && (weight_bytes >> s.xs) > (2 << 20) && s.tiles_m >= (8 >> s.xs)) ++s.xs;
    s.gs = 3 - s.xs;
    s.bn = tiles_n >> s.xs;
    s.bn_magic = udiv_magic(s.bn);
    const int64_t run = ((int64_t)s.tiles_m * s.bn + (1 << s.gs) - 1) >> s.gs;
    const int most = 32 * GL::UNIT;                       // workgroups that an XCD holds
    s.per_xcd = (int32_t)(run < most ? run : most);
    auto kern = gated_stream_kernel<ACT, BM, BF, TAIL>;
    static bool attr_done = false;
    if (!attr_done) {
        IBERT_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, GL::LDS));
        attr_done = true;
    }
    hipLaunchKernelGGL(kern, dim3(8u * (unsigned)s.per_xcd), dim3(64 * GL::NW), GL::LDS, stream, s);
    IBERT_LAUNCH_CHECK("gated_stream_kernel");
    static const KernelName name("gated_stream_kernel<%d, %d, %d, %s>", ACT, BM, BF, TAIL ? "true" : "false");
    g_last_kernel = name.text;
    return IBERT_OK;
}

int launch_gated_stream(const ibert_gated_desc& d, const int8_t* A, const int8_t* W, const int32_t* bias, const int32_t* mult, const int32_t* shift, int8_t* C, int tile,
                        hipStream_t stream)
{
    GatedStreamArgs s{};
    s.A = A; s.W = W; s.bias = bias; s.mult = mult; s.shift = shift; s.C = C;
    s.M = d.M; s.F = d.F; s.K = d.K; s.nk = (d.K + 127) / 128;
    s.lda = (int32_t)d.lda; s.ldw = (int32_t)d.ldw; s.ldc = (int32_t)d.ldc;
    const ibert_gate_params& p = d.gate;
    s.gate = gate_const(p);
    const bool gelu = !s.gate.silu, gelu_fast = gelu && gelu_fast_ok(p.gelu);
    s.fast = (int64_t)d.K * 16384 < (1 << 30) && p.out_dy.s >= 32 && p.out_dy.s <= 62 && (!gelu || gelu_fast);
    s.c_vec = aligned(C, 16) && d.ldc % 16 == 0;
    const int64_t w = 2 * (int64_t)d.F * d.K;
    auto launch = [&](auto act, auto bm, auto bf) {
        constexpr int ACT = decltype(act)::value, BM = decltype(bm)::value, BF = decltype(bf)::value;
        return d.K % 128 ? launch_gated_stream_as<ACT, BM, BF, true>(s, w, stream) : launch_gated_stream_as<ACT, BM, BF, false>(s, w, stream);
    };
    auto with = [&](auto bm, auto bf) {
        if (!gelu) return launch(std::integral_constant<int, GS_SILU>{}, bm, bf);
        if (gelu_fast && -2 * (int64_t)p.gelu.q_b < GatedLayout<decltype(bm)::value, decltype(bf)::value>::ERF) return launch(std::integral_constant<int, GS_GELU_TABLE>{}, bm, bf);
        return launch(std::integral_constant<int, GS_GELU>{}, bm, bf);
    };
    using std::integral_constant;
    if (tile == GATED_TALL) return with(integral_constant<int, 256>{}, integral_constant<int, 128>{});
    if (tile == GATED_LOW) return with(integral_constant<int, 128>{}, integral_constant<int, 128>{});
    return with(integral_constant<int, 128>{}, integral_constant<int, 64>{});
}

}  // namespace ibert
