// Products of few activation rows with weight matrices that are read once: 4-bit weights with group scales, and the INT8 weights of
// a gated block; plain (bias, requantization, residual) or ending in the gated product.
//
//   * The eight wavefronts of a workgroup share K in contiguous runs of chunks of 128, each for 8 BR rows and NT tiles of 16 channels, and work on their own until their
//     sums meet in LDS: integer sums, any order.
//   * 4-bit weights stand in memory as the matrix unit wants them: 1 KB a tile and chunk, 16 bytes a lane, whose low and high halves are the operands of two MFMAs.  A nibble
//     shifted to the top of its byte is 16 times its signed value, so that two operations on a dword unpack four weights, and the sums of a group (|sum| < 2^18) are shifted
//     back.
//   * sum_g s_g (sum_k a w - z_g sum_k a): the sum of a group's activations comes from an MFMA with ones, which leaves it in the lanes that need it.  Group terms are added
//     by 24-bit multiply-adds in 32 bits, which hold 4096 values of K (4096 * 128 * 15 * 255 < 2^31), then in 64.
//   * Activations past K are zeros: what weights hold there does not matter.
//   * Two kernels.  rows_ring_kernel: rows that are 16-byte aligned, K a multiple of 16; everything goes from memory straight into LDS, several chunks ahead.
//     rows_any_kernel: everything else, through registers, one chunk ahead.
//
// What bounds them (us with weights from memory / with three sets of them in turn, which the memory-side cache holds in part): for one row HBM (1 x 4096 -> 2 x 12288 in 4 bits,
// 51 MB: 11.8 / 10.3, 4.35 TB/s from memory), which takes several stages a wavefront and several workgroups a unit under way; for some ten rows instructions (16 x 1024 -> 50265
// 10.8 / 8.9, a wavefront has one chunk of K and its beginning and end beside it); for 64 the bytes that a unit has under way and what a block of rows reads again (64 x 12288 -> 4096
// 15.4 / 11.9).  rows_any_kernel: latency for few rows (5 x 2730 -> 1024 4.2), then one workgroup to a unit and one chunk ahead (2730 -> 4096: 33 rows 7.8, 256 25.7).
#pragma once
#include <type_traits>

#include "gate_math.h"

namespace ibert {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

struct RowsArgs {
    const int8_t* A;
    int64_t lda;
    int32_t M, N, K;               // N: output columns (of a gated block F)
    const void* w[2];              // INT8 rows, or packed 4-bit weights: [0] all or the gate's, [1] the up projection's
    const uint8_t* scales[2];
    const int8_t* zeros[2];
    int64_t ldw;
    const int32_t* bias;
    const int32_t* mult;
    const int32_t* shift;
    const int8_t* R;
    int64_t ldr;
    int32_t res_m, res_s;
    void* C;
    int64_t ldc;
    int32_t out_dtype, out_clamp;
    GateConst gate;
    int32_t chunks, per;           // chunks of 128 in K; of a wavefront's run
    int32_t stages;                // of a wavefront's ring
    int32_t a_vec, w_vec;          // rows of A, of INT8 weights are 16-byte aligned and K is a multiple of 16
    int32_t across, down;          // workgroups over the channels and over the rows
    uint32_t down_magic;           // see udiv_fix
};

constexpr int ROWS_THREADS = 512;

// 16 bytes of a row of n bytes at p from byte k on, zeros past its end; any alignment (memory is read unaligned here).  The last bytes of a row are moved down from its last 16:
// byte by byte they take as many trips to memory.
__device__ __forceinline__ v4i bytes_16(const int8_t* p, int k, int n)
{
    union { v4i v; uint64_t h[2]; int8_t b[16]; } u;
    if (k + 16 <= n) {
        __builtin_memcpy(u.b, p + k, 16);
        return u.v;
    }
    u.v = v4i{0, 0, 0, 0};
    if (k >= n) return u.v;
    if (n >= 16) {
        __builtin_memcpy(u.b, p + n - 16, 16);
        const int s = 8 * (k + 16 - n);                            // 8 .. 120
        if (s >= 64) u.h[0] = u.h[1] >> (s - 64);
        else u.h[0] = u.h[0] >> s | u.h[1] << (64 - s);
        u.h[1] = s >= 64 ? 0 : u.h[1] >> s;
        return u.v;
    }
    for (int i = 0; i < 16; ++i)
        if (k + i < n) u.b[i] = p[k + i];
    return u.v;
}

// Every argument in registers from here on, after one trip to memory: fetched where each is first used, behind branches, they are five.
template <bool W4, bool ZERO, bool GATED>
__device__ __forceinline__ void rows_arguments(const RowsArgs& g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" :: "s"(g.A), "s"(g.lda), "s"(g.M), "s"(g.N), "s"(g.K), "s"(g.w[0]), "s"(g.bias), "s"(g.mult), "s"(g.shift), "s"(g.C), "s"(g.ldc), "s"(g.chunks),
                 "s"(g.per), "s"(g.across), "s"(g.down), "s"(g.down_magic));
    if constexpr (W4) asm volatile("" :: "s"(g.scales[0]), "s"(g.stages));
    else asm volatile("" :: "s"(g.ldw), "s"(g.stages));
    if constexpr (W4 && GATED) asm volatile("" :: "s"(g.w[1]), "s"(g.scales[1]));
    if constexpr (ZERO) asm volatile("" :: "s"(g.zeros[0]), "s"(g.zeros[1]));
    if constexpr (GATED) asm volatile("" :: "s"(g.gate.silu), "s"(g.gate.m), "s"(g.gate.s), "s"(g.gate.gelu.q_b), "s"(g.gate.gelu.q_c), "s"(g.gate.gelu.q_1), "s"(g.gate.gelu.q_max),
                                   "s"(g.gate.gelu.m), "s"(g.gate.gelu.s));
    else asm volatile("" :: "s"(g.R), "s"(g.ldr), "s"(g.res_m), "s"(g.res_s), "s"(g.out_dtype), "s"(g.out_clamp));
#endif
}

// acc += the products of a chunk: activations xa (two halves of the chunk), packed weights w of NT tiles, their scales and zero points.
template <int MT, int NT, int G, bool ZERO>
__device__ __forceinline__ void chunk_products(v4i (&acc)[MT][NT], const v4i (&xa)[2][MT], const v4i (&w)[NT], const uint32_t (&sc)[NT], const uint32_t (&zc)[NT])
{
    constexpr int GPC = 128 / G;
    const v4i zero = {0, 0, 0, 0};
    // the sums of one group's products (or of its activations): group gi of the chunk, operands lo | hi
    auto group = [&](int j, int gi, const v4i& lo, const v4i& hi) {
        if (G == 128)
            return __builtin_amdgcn_mfma_i32_16x16x64_i8(xa[1][j], hi, __builtin_amdgcn_mfma_i32_16x16x64_i8(xa[0][j], lo, zero, 0, 0, 0), 0, 0, 0);
        if (G == 64) return __builtin_amdgcn_mfma_i32_16x16x64_i8(xa[gi & 1][j], gi & 1 ? hi : lo, zero, 0, 0, 0);
        const v4i x = xa[gi >> 1][j], y = gi & 2 ? hi : lo;
        const int e = 2 * (gi & 1);
        const long xl = (long)(((uint64_t)(uint32_t)x[e + 1] << 32) | (uint32_t)x[e]), yl = (long)(((uint64_t)(uint32_t)y[e + 1] << 32) | (uint32_t)y[e]);
        return __builtin_amdgcn_mfma_i32_16x16x32_i8(xl, yl, zero, 0, 0, 0);
    };
    v4i sa[MT][GPC];
    if constexpr (ZERO) {
        constexpr int ONES = 0x01010101;
        const v4i ones = {ONES, ONES, ONES, ONES};
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int gi = 0; gi < GPC; ++gi) sa[j][gi] = group(j, gi, ones, ones);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        v4i lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = (int)(((uint32_t)w[t][e] << 4) & 0xf0f0f0f0u);
            hi[e] = (int)((uint32_t)w[t][e] & 0xf0f0f0f0u);
        }
#pragma unroll
        for (int gi = 0; gi < GPC; ++gi) {
            const int32_t s = (int32_t)((sc[t] >> (8 * gi)) & 255u);
            int32_t z = 0;
            if constexpr (ZERO) z = (int32_t)(zc[t] << (28 - 8 * gi)) >> 28;           // (four bits, signed)
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const v4i p = group(j, gi, lo, hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    int32_t d = p[e] >> 4;
                    if constexpr (ZERO) d -= smul24(z, sa[j][gi][e]);
                    acc[j][t][e] = smad24(s, d, acc[j][t][e]);
                }
            }
        }
    }
}

struct RowsChannel {
    int32_t b, m, s;
};
__device__ __forceinline__ RowsChannel rows_channel(const RowsArgs& g, int ch)
{
    const uint32_t at = 4u * (uint32_t)ch;                         // (below 2^27: 32-bit offsets from the arrays' first entries)
    auto entry = [&](const int32_t* p) { return *reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(p) + at); };
    return RowsChannel{g.bias ? entry(g.bias) : 0, entry(g.mult), entry(g.shift)};
}

// Output (m, n) from its sums (of a gated block: gate and up projection), its channels' constants and its residual.
template <bool GATED>
__device__ __forceinline__ void rows_finish(const RowsArgs& g, int m, int n, int64_t s0, int64_t s1, const RowsChannel& c0, const RowsChannel& c1, int32_t res)
{
    const int64_t off = (int64_t)m * g.ldc + n;
    if constexpr (GATED) {
        static_cast<int8_t*>(g.C)[off] = (int8_t)gate_one(into_32(s0 + c0.b), into_32(s1 + c1.b), c0.m, c0.s, c1.m, c1.s, g.gate);
    } else {
        int64_t v = dy64(into_32(s0 + c0.b), c0.m, c0.s);
        if (g.R) v += dy64(res, g.res_m, g.res_s);
        const int32_t y = into(v, g.out_clamp);
        if (g.out_dtype == IBERT_I8) static_cast<int8_t*>(g.C)[off] = (int8_t)y;
        else if (g.out_dtype == IBERT_I16) static_cast<int16_t*>(g.C)[off] = (int16_t)y;
        else static_cast<int32_t*>(g.C)[off] = y;
    }
}

// INT8 sums have 32 bits, and so has what the biases make of them.
__device__ __forceinline__ void wrap_32(int64_t& s0, int64_t& s1, RowsChannel& c0, RowsChannel& c1)
{
    s0 = (int32_t)((uint32_t)s0 + (uint32_t)c0.b);
    s1 = (int32_t)((uint32_t)s1 + (uint32_t)c1.b);
    c0.b = c1.b = 0;
}

//   * Each wavefront has a ring of stages of its own in LDS -- 1 KB blocks of eight rows of A by 128 bytes, and of a tile's chunk of weights -- into which it requests
//     straight from memory as many chunks ahead as LDS holds; scales (and zero points) of its whole run come first.  The sums (a run is at most 4096 values: 32 bits) meet in LDS at the end.
//   * A's 16-byte units are swizzled by the row (see swz in gemm_kernel.h); a lane's operand is two reads of eight bytes, 32 apart.
// W4: 4-bit weights in groups of G (ZERO: with zero points), else INT8 rows.  BR: blocks of eight rows (1, 2, 4 or 8).  GATED: NT / 2 tiles of gate channels, then as many of the
// up projection.
template <bool W4, int BR, int NT, int G, bool ZERO, bool GATED>
__global__ __launch_bounds__(ROWS_THREADS) void rows_ring_kernel(RowsArgs g)
{
    // (blocks of a tile's chunk of weights: 1, or 2 of eight INT8 rows; requests of a chunk)
    constexpr int WB = W4 ? 1 : 2, NL = BR + WB * NT, STAGE = NL * 1024;
    constexpr int MT = (BR + 1) / 2, NH = GATED ? NT / 2 : NT, GPC = W4 ? 128 / G : 0;
    constexpr int TM = 8 * BR, PITCH = 16 * NT + 4;                // rows of the tile; dwords of a row of sums
    constexpr int EP = (TM * 16 * NH + ROWS_THREADS - 1) / ROWS_THREADS;
    constexpr int SUMS = TM * PITCH * 4;                           // bytes of a wavefront's sums, where its stages were
    static_assert(3 * NL < 64, "outstanding requests");
    extern __shared__ __align__(16) int8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, q = lane >> 4;
    rows_arguments<W4, ZERO, GATED>(g);
    const int jb = blockIdx.x >> 3, jc = udiv_fix(jb, g.down, g.down_magic), bx = jc * 8 + (blockIdx.x & 7);
    if (bx >= g.across) return;
    const int m0 = (jb - jc * g.down) * TM, rows = min(TM, g.M - m0), n0 = bx * (16 * NH);
    const int per = g.per, c0 = wave * per, run = min(per, g.chunks - c0);           // this wavefront's chunks [c0, c0 + run)
    const int stages = g.stages, scb = (per * 16 * GPC + 255) & ~255;                       // bytes of a tile's scales
    const int own = (ZERO ? 2 : 1) * NT * scb + max(stages * STAGE, SUMS);
    int8_t* const home = lds + wave * own;
    const uint32_t home0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t*)lds + (uint32_t)(wave * own);
    const uint32_t ring0 = home0 + (uint32_t)((ZERO ? 2 : 1) * NT * scb);
    int8_t* const ring = home + (ZERO ? 2 : 1) * NT * scb;

    // what the epilogue needs of its outputs' channels, behind the first requests: an output a thread and round
    RowsChannel ch[EP][GATED ? 2 : 1];
    int32_t res[EP];
    auto ends = [&]() {
#pragma unroll
        for (int p = 0; p < EP; ++p) {
            const int i = p * ROWS_THREADS + tid, m = i / (16 * NH), n = min(n0 + i - m * (16 * NH), g.N - 1);
            res[p] = 0;
            if (m < rows) {
                ch[p][0] = rows_channel(g, n);
                if constexpr (GATED) ch[p][1] = rows_channel(g, g.N + n);
                if (!GATED && g.R) res[p] = g.R[(int64_t)(m0 + m) * g.ldr + n];
            }
        }
    };
    if (run <= 0) ends();
    else {
        const uint8_t* wp[W4 ? NT : 1];
        const int64_t tbytes = (int64_t)g.chunks * 1024;
        // (tiles past the last channel read the last one again)
        auto tile_of = [&](int t) { return min(n0 + 16 * (t % NH), g.N - 1) >> 4; };
        if constexpr (W4) {
#pragma unroll
            for (int t = 0; t < NT; ++t) wp[t] = static_cast<const uint8_t*>(g.w[t / NH]) + tile_of(t) * tbytes;
        }
        // scales of the run, 64 dwords a request; what lies past the tile's last reads as zeros
        auto buffer = [](const void* p, uint32_t bytes) {
            const uint64_t u = (uint64_t)(uintptr_t)p;
            return v4i{(int32_t)(uint32_t)u, (int32_t)((uint32_t)(u >> 32) & 0xffffu), (int32_t)bytes, 0x00020000};
        };
        const uint32_t sbytes = (uint32_t)(g.chunks * 16 * GPC);
#pragma unroll
        for (int t = 0; t < (W4 ? NT : 0); ++t)
#pragma unroll
            for (int z = 0; z < (ZERO ? 2 : 1); ++z) {
                const void* src = z ? static_cast<const void*>(g.zeros[t / NH]) : static_cast<const void*>(g.scales[t / NH]);
                const v4i d = buffer(static_cast<const uint8_t*>(src) + (int64_t)tile_of(t) * sbytes, sbytes);
                for (int k = 0; k < scb; k += 256)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                                 :: "s"(home0 + (uint32_t)((z * NT + t) * scb + k)), "v"((uint32_t)(c0 * 16 * GPC + k + 4 * lane)), "s"(d) : "memory", "m0");
            }
        // requests of a chunk: BR blocks of A (rows past the last read that one again; bytes past K zeros), NT of weights
        const v4i da = buffer(g.A + (int64_t)m0 * g.lda, (uint32_t)((rows - 1) * (int)g.lda + g.K));
        const int lr8 = lane >> 3, lp = lane & 7;
        const int unit0 = lp ^ (lr8 >> 1), unit1 = unit0 ^ 4;
        uint32_t va[BR];
#pragma unroll
        for (int b = 0; b < BR; ++b) va[b] = (uint32_t)(min(8 * b + lr8, rows - 1) * (int)g.lda + (b & 1 ? unit1 : unit0) * 16);
        const int left0 = g.K - unit0 * 16, left1 = g.K - unit1 * 16;
        // INT8 weights: blocks of eight rows as those of A, channels past the last as that one again
        v4i dw[W4 ? 1 : NT];
        uint32_t vw[W4 ? 1 : 2 * NT];
        if constexpr (!W4) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int first = min(n0 + 16 * (t % NH), g.N - 1), left = min(16, g.N - first);
                dw[t] = buffer(static_cast<const int8_t*>(g.w[0]) + ((int64_t)(t / NH) * g.N + first) * g.ldw, (uint32_t)((left - 1) * (int)g.ldw + g.K));
#pragma unroll
                for (int b = 0; b < 2; ++b) vw[2 * t + b] = (uint32_t)(min(8 * b + lr8, left - 1) * (int)g.ldw + (b ? unit1 : unit0) * 16);
            }
        }
        auto request = [&](int chunk, int st) {
            const int c = __builtin_amdgcn_readfirstlane(chunk);   // (the same in every lane: the compiler loses sight of it)
            const uint32_t to = (uint32_t)__builtin_amdgcn_readfirstlane((int)ring0 + st * STAGE);
#pragma unroll
            for (int b = 0; b < BR; ++b)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                             :: "s"(to + (uint32_t)(b * 1024)), "v"(c * 128 < (b & 1 ? left1 : left0) ? va[b] + (uint32_t)(c * 128) : 0xfffffff0u), "s"(da)
                             : "memory", "m0");
            if constexpr (W4) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                                 :: "s"(to + (uint32_t)((BR + t) * 1024)), "v"((uint32_t)lane * 16u), "s"(wp[t] + (int64_t)c * 1024) : "memory", "m0");
            } else {
#pragma unroll
                for (int b = 0; b < 2 * NT; ++b)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                                 :: "s"(to + (uint32_t)((BR + b) * 1024)), "v"(c * 128 < (b & 1 ? left1 : left0) ? vw[b] + (uint32_t)(c * 128) : 0xfffffff0u), "s"(dw[b / 2])
                                 : "memory", "m0");
            }
        };
        for (int i = 0; i < stages; ++i)
            if (i < run) request(c0 + i, i);
        ends();

        v4i acc[MT][NT];
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[j][t] = v4i{0, 0, 0, 0};
        constexpr auto vm = [](int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); };
        const int ra = BR == 1 ? r & 7 : r;
        const int a0 = ra * 128 + (((q >> 1) ^ ((ra >> 1) & 7)) << 4) + (q & 1) * 8;
        const int a8 = ra * 128 + ((q ^ ((ra >> 1) & 7)) << 4), w8 = r * 128 + ((q ^ ((r >> 1) & 7)) << 4);
        int st = 0;
        for (int i = 0; i < run; ++i) {
            const int younger = min(run - 1 - i, stages - 1);
            if (younger == 0) __builtin_amdgcn_s_waitcnt(vm(0));
            else if (younger == 1) __builtin_amdgcn_s_waitcnt(vm(NL));
            else if (younger == 2) __builtin_amdgcn_s_waitcnt(vm(2 * NL));
            else __builtin_amdgcn_s_waitcnt(vm(3 * NL));
            asm volatile("" ::: "memory");
            const int8_t* const base = ring + st * STAGE;
            v4i xa[2][MT];
            if constexpr (!W4) {
                v4i w[2][NT];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int j = 0; j < MT; ++j) xa[h][j] = *reinterpret_cast<const v4i*>(base + j * 2048 + (a8 ^ (h * 64)));
#pragma unroll
                    for (int t = 0; t < NT; ++t) w[h][t] = *reinterpret_cast<const v4i*>(base + (BR + 2 * t) * 1024 + (w8 ^ (h * 64)));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < MT; ++j) acc[j][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(xa[h][j], w[h][t], acc[j][t], 0, 0, 0);
            } else {
                v4i w[NT];
                uint32_t sc[NT], zc[NT];
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    // (the rows' addresses apart: read in pairs of rows the operands would have to be put together by moves)
                    int aj = a0 + j * 2048;
                    asm volatile("" : "+v"(aj));
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const v2i lo = *reinterpret_cast<const v2i*>(base + (aj ^ (h * 64))), hi = *reinterpret_cast<const v2i*>(base + (aj ^ (h * 64 + 32)));
                        xa[h][j] = v4i{lo[0], lo[1], hi[0], hi[1]};
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    w[t] = *reinterpret_cast<const v4i*>(base + (BR + t) * 1024 + lane * 16);
                    auto scale = [&](const int8_t* p) {
                        p += (i * 16 + r) * GPC;
                        return GPC == 4 ? *reinterpret_cast<const uint32_t*>(p) : (GPC == 2 ? *reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint8_t*>(p));
                    };
                    sc[t] = scale(home + t * scb);
                    if constexpr (ZERO) zc[t] = scale(home + (NT + t) * scb);
                }
                chunk_products<MT, NT, G, ZERO>(acc, xa, w, sc, zc);
            }
            if (i + stages < run) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage has been read
                request(c0 + i + stages, st);
            }
            st = st + 1 == stages ? 0 : st + 1;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        int32_t* const sums = reinterpret_cast<int32_t*>(ring);
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (BR > 1 || q < 2) sums[(16 * j + 4 * q + e) * PITCH + 16 * t + r] = acc[j][t][e];
    }
    __syncthreads();

    // ---- epilogue: an output a thread and round
    const int runs = (g.chunks + per - 1) / per;
#pragma unroll
    for (int p = 0; p < EP; ++p) {
        const int i = p * ROWS_THREADS + tid, m = i / (16 * NH), nn = i - m * (16 * NH), n = n0 + nn;
        if (m >= rows || n >= g.N) continue;
        const int8_t* const at = lds + (ZERO ? 2 : 1) * NT * scb + (m * PITCH + nn) * 4;
        // (of INT8 weights, and of up to 4096 values of K, all of a sum has 32 bits)
        int64_t s0 = 0, s1 = 0;
        auto add = [&](auto zero) {
            auto t0 = zero, t1 = zero;
#pragma unroll
            for (int w = 0; w < 8; ++w)
                if (w < runs) {
                    t0 += *reinterpret_cast<const int32_t*>(at + w * own);
                    if constexpr (GATED) t1 += *reinterpret_cast<const int32_t*>(at + w * own + 64 * NH);
                }
            s0 = W4 ? (int64_t)t0 : (int64_t)(int32_t)t0;
            s1 = W4 ? (int64_t)t1 : (int64_t)(int32_t)t1;
        };
        if (!W4) add(0u);
        else if (g.K <= 4096) add(0);
        else add((int64_t)0);
        if constexpr (!W4) wrap_32(s0, s1, ch[p][0], ch[p][GATED ? 1 : 0]);
        rows_finish<GATED>(g, m0 + m, n, s0, s1, ch[p][0], ch[p][GATED ? 1 : 0], res[p]);
    }
}

// Rows of any alignment, any K.  A wavefront's next chunk is on its way into registers while it multiplies this one, whose rows pass through LDS (their units swizzled as in
// rows_ring_kernel; 4-bit weights need not).  Sums of 4-bit weights go to 64 bits in LDS every 32 chunks.
template <bool W4, int BR, int NT, int G, bool ZERO, bool GATED>
__global__ __launch_bounds__(ROWS_THREADS) void rows_any_kernel(RowsArgs g)
{
    typedef std::conditional_t<W4, int64_t, int32_t> sum_t;
    constexpr int MT = (BR + 1) / 2, NH = GATED ? NT / 2 : NT, GPC = W4 ? 128 / G : 1, WB = W4 ? 1 : 2, TM = 8 * BR, PITCH = 16 * NT + 4;
    constexpr int EP = (TM * 16 * NH + ROWS_THREADS - 1) / ROWS_THREADS;
    constexpr int STAGE = (BR + (W4 ? 0 : 2 * NT)) * 1024, SUMS = TM * PITCH * (int)sizeof(sum_t);
    // (sums of INT8 weights go, at the end, where the stage was)
    constexpr int SUMS_AT = W4 ? STAGE : 0, OWN = W4 ? STAGE + SUMS : (STAGE > SUMS ? STAGE : SUMS);
    extern __shared__ __align__(16) int8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, q = lane >> 4;
    rows_arguments<W4, ZERO, GATED>(g);
    const int jb = blockIdx.x >> 3, jc = udiv_fix(jb, g.down, g.down_magic), bx = jc * 8 + (blockIdx.x & 7);
    if (bx >= g.across) return;
    const int m0 = (jb - jc * g.down) * TM, rows = min(TM, g.M - m0), n0 = bx * (16 * NH);
    const int per = g.per, c0 = wave * per, run = min(per, g.chunks - c0);
    int8_t* const stage = lds + wave * OWN;
    sum_t* const sums = reinterpret_cast<sum_t*>(stage + SUMS_AT);
    // what the epilogue needs of its outputs' channels, behind the first loads: an output a thread and round
    RowsChannel ch[EP][GATED ? 2 : 1];
    int32_t res[EP];
    auto ends = [&]() {
#pragma unroll
        for (int p = 0; p < EP; ++p) {
            const int i = p * ROWS_THREADS + tid, m = i / (16 * NH), n = min(n0 + i - m * (16 * NH), g.N - 1);
            res[p] = 0;
            if (m < rows) {
                ch[p][0] = rows_channel(g, n);
                if constexpr (GATED) ch[p][1] = rows_channel(g, g.N + n);
                if (!GATED && g.R) res[p] = g.R[(int64_t)(m0 + m) * g.ldr + n];
            }
        }
    };
    if (run <= 0) ends();
    else {
        const int lr8 = lane >> 3, lp = lane & 7;
        auto tile_of = [&](int t) { return min(n0 + 16 * (t % NH), g.N - 1) >> 4; };
        struct Chunk {
            v4i a[BR], w[WB * NT];
            uint32_t s[NT], z[NT];
        };
        auto load = [&](int c, Chunk& x) {
#pragma unroll
            for (int b = 0; b < BR; ++b) x.a[b] = bytes_16(g.A + (int64_t)(m0 + min(8 * b + lr8, rows - 1)) * g.lda, c * 128 + 16 * lp, g.K);
            if constexpr (W4) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int64_t at = (int64_t)tile_of(t) * g.chunks + c;
                    x.w[t] = *reinterpret_cast<const v4i*>(static_cast<const uint8_t*>(g.w[t / NH]) + at * 1024 + lane * 16);
                    auto scale = [&](const void* base) {
                        const uint8_t* p = static_cast<const uint8_t*>(base) + (at * 16 + r) * GPC;
                        return GPC == 4 ? *reinterpret_cast<const uint32_t*>(p) : (GPC == 2 ? *reinterpret_cast<const uint16_t*>(p) : *p);
                    };
                    x.s[t] = scale(g.scales[t / NH]);
                    if constexpr (ZERO) x.z[t] = scale(g.zeros[t / NH]);
                }
            } else {
#pragma unroll
                for (int b = 0; b < 2 * NT; ++b) {
                    const int n = min(n0 + 16 * (b / 2 % NH) + 8 * (b & 1) + lr8, g.N - 1);
                    x.w[b] = bytes_16(static_cast<const int8_t*>(g.w[0]) + ((int64_t)(b / 2 / NH) * g.N + n) * g.ldw, c * 128 + 16 * lp, g.K);
                }
            }
        };
        v4i acc[MT][NT];
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[j][t] = v4i{0, 0, 0, 0};
        // (its own lanes read and write them: no other wavefront does before the barrier)
        auto keep = [&](bool first) {
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (BR > 1 || q < 2) {
                            sum_t& s = sums[(16 * j + 4 * q + e) * PITCH + 16 * t + r];
                            s = (first ? 0 : s) + acc[j][t][e];
                        }
                    acc[j][t] = v4i{0, 0, 0, 0};
                }
        };
        // where the lane's 16 bytes of a block go, and where its operands are
        const int to0 = lr8 * 128 + ((lp ^ (lr8 >> 1)) << 4), ra = BR == 1 ? r & 7 : r;
        const int a0 = ra * 128 + (((q >> 1) ^ ((ra >> 1) & 7)) << 4) + (q & 1) * 8;
        const int a8 = ra * 128 + ((q ^ ((ra >> 1) & 7)) << 4), w8 = r * 128 + ((q ^ ((r >> 1) & 7)) << 4);
        Chunk x;
        load(c0, x);
        ends();
        for (int i = 0; i < run; ++i) {
#pragma unroll
            for (int b = 0; b < BR; ++b) *reinterpret_cast<v4i*>(stage + b * 1024 + (b & 1 ? to0 ^ 64 : to0)) = x.a[b];
            v4i w[NT];
            uint32_t sc[NT], zc[NT];
            if constexpr (W4) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    w[t] = x.w[t];
                    sc[t] = x.s[t];
                    if constexpr (ZERO) zc[t] = x.z[t];
                }
            } else {
#pragma unroll
                for (int b = 0; b < 2 * NT; ++b) *reinterpret_cast<v4i*>(stage + (BR + b) * 1024 + (b & 1 ? to0 ^ 64 : to0)) = x.w[b];
            }
            if (i + 1 < run) load(c0 + i + 1, x);
            v4i xa[2][MT];
            if constexpr (W4) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < MT; ++j) {
                        const v2i lo = *reinterpret_cast<const v2i*>(stage + j * 2048 + (a0 ^ (h * 64))), hi = *reinterpret_cast<const v2i*>(stage + j * 2048 + (a0 ^ (h * 64 + 32)));
                        xa[h][j] = v4i{lo[0], lo[1], hi[0], hi[1]};
                    }
                chunk_products<MT, NT, G, ZERO>(acc, xa, w, sc, zc);
                if ((i & 31) == 31) keep(i == 31);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v4i wb[NT];
#pragma unroll
                    for (int j = 0; j < MT; ++j) xa[h][j] = *reinterpret_cast<const v4i*>(stage + j * 2048 + (a8 ^ (h * 64)));
#pragma unroll
                    for (int t = 0; t < NT; ++t) wb[t] = *reinterpret_cast<const v4i*>(stage + (BR + 2 * t) * 1024 + (w8 ^ (h * 64)));
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < MT; ++j) acc[j][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(xa[h][j], wb[t], acc[j][t], 0, 0, 0);
                }
            }
        }
        keep(!W4 || run < 32);
    }
    __syncthreads();

    const int runs = (g.chunks + per - 1) / per;
#pragma unroll
    for (int p = 0; p < EP; ++p) {
        const int i = p * ROWS_THREADS + tid, m = i / (16 * NH), nn = i - m * (16 * NH), n = n0 + nn;
        if (m >= rows || n >= g.N) continue;
        int64_t s0 = 0, s1 = 0;
        for (int w = 0; w < runs; ++w) {
            const sum_t* const at = reinterpret_cast<const sum_t*>(lds + w * OWN + SUMS_AT) + m * PITCH + nn;
            s0 += at[0];
            if constexpr (GATED) s1 += at[16 * NH];
        }
        if constexpr (!W4) wrap_32(s0, s1, ch[p][0], ch[p][GATED ? 1 : 0]);
        rows_finish<GATED>(g, m0 + m, n, s0, s1, ch[p][0], ch[p][GATED ? 1 : 0], res[p]);
    }
}

}  // namespace ibert
