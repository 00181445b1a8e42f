// Logits of the vocabulary before Softmax or a choice: penalties for repeated tokens, biases, grammar masks.
//
// A workgroup takes a slice of one row's vocabulary.  It counts the row's tokens that fall into the slice, and adds up the biases there, in
// LDS (integer atomics: any order gives the same), then passes over the logits once.  The history is read once per slice, from L2.
// What bounds it (64 x 128000, 65.5 MB, us, inputs from memory): the logits' way through HBM, 14.8 without a history (4.4 TB/s with the launch).  A short history (up to 500 tokens a
// row) adds trips to memory, for where its tokens are and for the tokens, 17.6; a long one (up to 8191) instructions, 2.5 times those without: counting, and 64-bit penalties that a
// wavefront goes through where one of its lanes has a token seen, 21.4 (ALU slots 0.63, waits 0.20, four workgroups a unit).  22.1 with biases and masks; 18.4 with three sets of inputs in
// turn, which the memory-side cache holds in part.  Kept in registers for the next slice (workgroups that go through several slices) or dealt to wavefronts of their own, the loads
// cost so many registers that fewer workgroups fit: 35.7 and 42.4 us.
#include "common.h"

namespace ibert {

typedef int v4i __attribute__((ext_vector_type(4)));

struct LogitsArgs {
    const int32_t* x;
    int32_t* y;
    const ibert_logits_row* params;
    const int32_t* tokens;
    const int32_t* token_start;
    const int32_t* out_start;
    const int32_t* bias_ids;
    const int32_t* bias_values;
    const int32_t* bias_start;
    const uint32_t* masks;
    int64_t ldx, ldy;
    int32_t vocab, num_tokens, num_biases, num_masks, ld_mask;
    int32_t slices;                // of a row
    uint32_t slices_magic;         // see udiv_fix
    int32_t rows, by_xcd;          // of this launch; slices of a row all on one XCD
    int32_t vec;                   // rows allow 16-byte loads and stores
};

// Threads of a workgroup, tokens of its slice.  The logits of a slice (8 a thread) are requested first and arrive while the history is counted.
constexpr int LOGITS_THREADS = 512;
constexpr uint32_t SEEN = 0x80000000u, BIASED = 0x40000000u;     // in the prompt; has biases; the low bits count what has been produced

// Into INT32: the low half where the high one is its sign.
__device__ __forceinline__ int32_t saturated(int64_t v)
{
    const int32_t lo = (int32_t)v, hi = (int32_t)(v >> 32);
    return hi == lo >> 31 ? lo : (hi >> 31) ^ INT32_MAX;
}

// What a row does to a logit, its halves of rounding made once.
struct Penalty {
    int32_t up_m, up_s, down_m, down_s, presence, frequency;
    int64_t up_rnd, down_rnd;
};
__device__ __forceinline__ Penalty penalty_of(const ibert_logits_row& p)
{
    const int32_t us = clamp_i32(p.up.s, 0, 62), ds = clamp_i32(p.down.s, 0, 62);
    return Penalty{p.up.m, us, p.down.m, ds, p.presence, p.frequency, ((int64_t)1 << us) >> 1, ((int64_t)1 << ds) >> 1};
}

// count != 0
__device__ __forceinline__ int32_t adjusted(int32_t x, uint32_t count, int64_t bias, const Penalty& p)
{
    if (x == INT32_MIN) return x;
    const bool up = x > 0;
    const int64_t m = (int64_t)x * (up ? p.up_m : p.down_m) + (up ? p.up_rnd : p.down_rnd);
    const int32_t r = count & ~BIASED ? saturated(m >> (up ? p.up_s : p.down_s)) : x, n = (int32_t)(count & ~(SEEN | BIASED));
    const int32_t y = saturated((int64_t)r - (n ? p.presence : 0) - (int64_t)p.frequency * n + bias);
    return y == INT32_MIN ? INT32_MIN + 1 : y;
}

template <int LOGITS_SLICE>
__global__ __launch_bounds__(LOGITS_THREADS, 8) void logits_adjust_kernel(LogitsArgs g)
{
    extern __shared__ __align__(16) int32_t room[];
    // workgroups go round the XCDs: with many rows each XCD takes every eighth, whose tokens then come into one L2 and not into eight
    const int tid = threadIdx.x, id = g.by_xcd ? (int)(blockIdx.x >> 3) : (int)blockIdx.x, part = udiv_fix(id, g.slices, g.slices_magic);
    const int row = g.by_xcd ? 8 * part + (int)(blockIdx.x & 7) : part, t0 = (id - part * g.slices) * LOGITS_SLICE;
    if (row >= g.rows) return;
    const int n = min(LOGITS_SLICE, g.vocab - t0);
    uint32_t* const count = reinterpret_cast<uint32_t*>(room);
    int32_t* const bias = room + LOGITS_SLICE;                      // where there are biases at all
    const ibert_logits_row p = g.params[row];
    int ts = 0, te = 0, made = 0, bs = 0, be = 0;
    if (g.num_tokens > 0) {
        ts = clamp_i32(g.token_start[row], 0, g.num_tokens);
        te = clamp_i32(g.token_start[row + 1], ts, g.num_tokens);
        made = clamp_i32(g.out_start[row], ts, te);
    }
    if (g.num_biases > 0) {
        bs = clamp_i32(g.bias_start[row], 0, g.num_biases);
        be = clamp_i32(g.bias_start[row + 1], bs, g.num_biases);
    }
    const bool biased = be > bs;
    // Sums of biases have 32 bits where every value in the slice is below 2^31 / (be - bs) in size, so that none can overflow; where one is not, the list is gone through
    // again with 64-bit sums, for half of the slice at a time in the same room.  (With 64 bits for every token at once a unit holds three workgroups in place of four.)
    // us, no such value in a row's list / one: 8 x 50265, 300 biases a row at most, 6.4 / 6.7; 64 x 128000, 300 22.3 / 23.0, 10000 35.3 / 42.7.
    const uint32_t small = biased ? 0x7fffffffu / (uint32_t)(be - bs) : 0;
    __shared__ int32_t wide;

    // Loads arrive in the order in which they are asked for: first what is counted, then the logits.  (The other way round nothing is counted before the
    // logits are there, and every workgroup takes two trips to memory one after the other: 64 x 128000 with 262 thousand tokens 26.5 / 24.9 us.)
    constexpr int LV = 4, ROUND = 4 * LV * LOGITS_THREADS;          // loads of four tokens under way; tokens of a round
    // four tokens from an aligned place on, none (-1) outside the row's; words of other rows are not read
    auto load4 = [&](int at) {
        v4i a = {-1, -1, -1, -1};
        if (at >= ts && at + 4 <= te) a = *reinterpret_cast<const v4i*>(g.tokens + at);
        else if (at + 4 > ts && at < te) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at + e >= ts && at + e < te) a[e] = g.tokens[at + e];
        }
        return a;
    };
    const int first = ts - (int)((reinterpret_cast<uintptr_t>(g.tokens + ts) >> 2) & 3) + 4 * tid;
    v4i a[LV];
#pragma unroll
    for (int k = 0; k < LV; ++k) a[k] = load4(first + 4 * k * LOGITS_THREADS);
    int32_t bid = -1, bval = 0;
    if (bs + tid < be) {
        bid = g.bias_ids[bs + tid];
        bval = g.bias_values[bs + tid];
    }
    const uint32_t* const mask = g.num_masks > 0 && p.mask >= 0 ? g.masks + (int64_t)min(p.mask, g.num_masks - 1) * g.ld_mask : nullptr;
    const int32_t* const x = g.x + (int64_t)row * g.ldx + t0;
    int32_t* const y = g.y + (int64_t)row * g.ldy + t0;
    constexpr int PER = LOGITS_SLICE / (4 * LOGITS_THREADS);
    v4i logits[PER];
    uint32_t words[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = 4 * (k * LOGITS_THREADS + tid);
        logits[k] = v4i{0, 0, 0, 0};
        words[k] = 0;
        if (g.vec && i + 4 <= n) {
            logits[k] = *reinterpret_cast<const v4i*>(x + i);
            if (mask) words[k] = mask[(t0 + i) >> 5];
        }
    }
    for (int i = 4 * tid; i < n; i += 4 * LOGITS_THREADS) {
        *reinterpret_cast<v4i*>(count + i) = v4i{0, 0, 0, 0};
        if (biased) *reinterpret_cast<v4i*>(bias + i) = v4i{0, 0, 0, 0};
    }
    if (tid == 0) wide = 0;
    __syncthreads();
    for (int i = first;; i += ROUND) {
#pragma unroll
        for (int k = 0; k < LV; ++k) {
            if (i + 4 * k * LOGITS_THREADS >= te) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t t = (uint32_t)a[k][e] - (uint32_t)t0;
                if (t < (uint32_t)n) {
                    if (i + 4 * k * LOGITS_THREADS + e >= made) atomicAdd(&count[t], 1u);
                    else atomicOr(&count[t], SEEN);
                }
            }
        }
        if (i + ROUND >= te) break;
#pragma unroll
        for (int k = 0; k < LV; ++k) a[k] = load4(i + ROUND + 4 * k * LOGITS_THREADS);
    }
    for (int i = bs + tid; i < be; i += LOGITS_THREADS) {
        if (i >= bs + LOGITS_THREADS) {
            bid = g.bias_ids[i];
            bval = g.bias_values[i];
        }
        const uint32_t t = (uint32_t)bid - (uint32_t)t0;
        if (t < (uint32_t)n) {
            atomicOr(&count[t], BIASED);
            atomicAdd(&bias[t], bval);
            if ((uint32_t)(bval < 0 ? 0u - (uint32_t)bval : (uint32_t)bval) > small) wide = 1;
        }
    }
    __syncthreads();
    const Penalty pen = penalty_of(p);
    auto one = [&](int i, int32_t v, uint32_t word, auto&& bias_of) {
        if (mask && !((word >> ((t0 + i) & 31)) & 1u)) return INT32_MIN;
        const uint32_t c = count[i];
        return c ? adjusted(v, c, c & BIASED ? (int64_t)bias_of(i) : 0, pen) : v;
    };
    if (biased && wide) {
        constexpr int HALF = LOGITS_SLICE / 2;
        unsigned long long* const sum = reinterpret_cast<unsigned long long*>(bias);
        for (int h = 0; h < n; h += HALF) {
            const int end = min(n, h + HALF);
            for (int i = tid; i < HALF; i += LOGITS_THREADS) sum[i] = 0;
            __syncthreads();
            for (int i = bs + tid; i < be; i += LOGITS_THREADS) {
                const uint32_t t = (uint32_t)g.bias_ids[i] - (uint32_t)(t0 + h);
                if (t < (uint32_t)(end - h)) atomicAdd(&sum[t], (unsigned long long)(int64_t)g.bias_values[i]);
            }
            __syncthreads();
            for (int i = h + tid; i < end; i += LOGITS_THREADS) y[i] = one(i, x[i], mask ? mask[(t0 + i) >> 5] : 0, [&](int j) { return (int64_t)sum[j - h]; });
            __syncthreads();
        }
        return;
    }
    auto narrow = [&](int i) { return bias[i]; };
    if (g.vec) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = 4 * (k * LOGITS_THREADS + tid);
            if (i + 4 > n) continue;
            v4i v = logits[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = one(i + e, v[e], words[k], narrow);
            *reinterpret_cast<v4i*>(y + i) = v;
        }
    }
    for (int i = (g.vec ? n & ~3 : 0) + tid; i < n; i += LOGITS_THREADS) y[i] = one(i, x[i], mask ? mask[(t0 + i) >> 5] : 0, narrow);
}

template <int LOGITS_SLICE>
static int launch_logits(LogitsArgs g, int64_t rows, hipStream_t stream)
{
    auto kern = logits_adjust_kernel<LOGITS_SLICE>;
    const size_t lds = (size_t)LOGITS_SLICE * (g.num_biases > 0 ? 8 : 4);
    g.slices = (g.vocab + LOGITS_SLICE - 1) / LOGITS_SLICE;
    g.slices_magic = udiv_magic(g.slices);
    // (a launch may have 2^32 threads at most: pieces of rows)
    const int64_t most = (1 << 22) / g.slices / 8 * 8;               // (at most 2^15 slices)
    for (int64_t r0 = 0; r0 < rows; r0 += most) {
        const int64_t n = rows - r0 < most ? rows - r0 : most;
        LogitsArgs a = g;
        a.x += r0 * g.ldx;
        a.y += r0 * g.ldy;
        a.params += r0;
        if (a.token_start) a.token_start += r0;
        if (a.out_start) a.out_start += r0;
        if (a.bias_start) a.bias_start += r0;
        a.rows = (int32_t)n;
        a.by_xcd = n % 8 == 0 || n >= 128;
        hipLaunchKernelGGL(kern, dim3((unsigned)((a.by_xcd ? (n + 7) / 8 * 8 : n) * g.slices)), dim3(LOGITS_THREADS), lds, stream, a);
        IBERT_LAUNCH_CHECK("logits_adjust_kernel");
    }
    static const KernelName name("logits_adjust_kernel<%d>", LOGITS_SLICE);
    g_last_kernel = name.text;
    return IBERT_OK;
}

}  // namespace ibert

extern "C" int ibert_logits_adjust_i(const ibert_logits_desc* desc, const int32_t* x, const ibert_logits_row* params, const int32_t* tokens,
                                     const int32_t* token_start, const int32_t* out_start, const int32_t* bias_ids, const int32_t* bias_values,
                                     const int32_t* bias_start, const uint32_t* masks, int32_t* y, void* stream)
{
    if (!desc) return IBERT_ERR_NULL;
    const ibert_logits_desc& d = *desc;
    if (d.rows < 0 || d.vocab < 0 || d.vocab > (1 << 26) || d.num_tokens < 0 || d.num_tokens >= (1 << 30) || d.num_biases < 0 || d.num_biases >= (1 << 30) ||
        d.num_masks < 0 || d.ldx < d.vocab || d.ldy < d.vocab || (d.num_masks > 0 && d.ld_mask < (d.vocab + 31) / 32)) return IBERT_ERR_SHAPE;
    if (d.rows == 0 || d.vocab == 0) return IBERT_OK;
    if (!x || !y || !params || (d.num_tokens > 0 && (!tokens || !token_start || !out_start)) ||
        (d.num_biases > 0 && (!bias_ids || !bias_values || !bias_start)) || (d.num_masks > 0 && !masks)) return IBERT_ERR_NULL;
    typedef unsigned __int128 extent;                              // (whatever leading dimensions are given)
    const extent px = reinterpret_cast<uintptr_t>(x), py = reinterpret_cast<uintptr_t>(y);
    const extent sx = 4 * ((extent)(d.rows - 1) * (extent)d.ldx + d.vocab), sy = 4 * ((extent)(d.rows - 1) * (extent)d.ldy + d.vocab);
    if (!(px == py && d.ldx == d.ldy) && px < py + sy && py < px + sx) return IBERT_ERR_SHAPE;
    ibert::LogitsArgs g{};
    g.x = x; g.y = y; g.params = params;
    if (d.num_tokens > 0) { g.tokens = tokens; g.token_start = token_start; g.out_start = out_start; }
    if (d.num_biases > 0) { g.bias_ids = bias_ids; g.bias_values = bias_values; g.bias_start = bias_start; }
    g.masks = masks;
    g.ldx = d.ldx; g.ldy = d.ldy;
    g.vocab = d.vocab; g.num_tokens = d.num_tokens; g.num_biases = d.num_biases; g.num_masks = d.num_masks; g.ld_mask = d.ld_mask;
    g.vec = ibert::aligned(x, 16) && ibert::aligned(y, 16) && d.ldx % 4 == 0 && d.ldy % 4 == 0;
    // Slices of 4096, or of 2048 where the longer ones would not be two workgroups to a unit.  us with inputs from memory, 2048 / 4096 (8192): 1 x 50265 4.0 / 5.0 (6.6), 64 x 128000 with 262 thousand
    // tokens and 10 thousand biases 26.6 / 22.7 (25.9), without any 18.7 / 16.0 (16.1).
    if ((int64_t)d.rows * ((d.vocab + 4095) / 4096) < 512) return ibert::launch_logits<2048>(g, d.rows, static_cast<hipStream_t>(stream));
    return ibert::launch_logits<4096>(g, d.rows, static_cast<hipStream_t>(stream));
}
