// Rotary positions of queries and keys, the optional norm of each head in front of them, and the append of keys and values to
// the paged cache (ibert_rotary_append_i): one launch over the packed QKV rows, in which some workgroups take queries, some keys,
// some values.
//
// Queries and keys: a head takes D / 2P lanes, each the two halves of P pairs, so that no value crosses lanes for the rotation.
// (Half layout: channels P j .. and P j + R/2 ..; interleaved, and behind the rotated part: 2P j .. and 2P j + P ..)  P = 16 where
// whole pieces of 16 bytes come out of it (R a multiple of 32), else 8.  The norm adds up squares over the head's lanes in
// registers.  Cosine and sine stand in a table with 14 fractional bits: a rotated value is below 2^30, and its requantization is the
// same 64-bit step as a MatMul's.
// Values: the cache wants 16 tokens of a channel side by side.  A wavefront takes 16 channels of 64 rows.  Where rows follow each other into
// a block of 64 tokens (a prompt), their bytes are transposed, four rows by lane swaps and the rest through LDS, and leave as 1 KB, or
// as the dwords and bytes of it that they fill; single rows are stored byte by byte.
// Bound: HBM, and with norms the vector ALU next to it.  16384 rows of 32 + 8 + 8 heads of width 128: 206 MB in 49 us without norms (4.2 TB/s), in 61 us with them
// (3.4 TB/s; 0.79 of the ALU's slots).  2741 rows of 16 + 16 + 16 heads of width 64: 17 MB in 7.6 us.  Five rows: 3.5 us, three dependent trips to memory.
#include "layernorm_math.h"
#include "ibert_testing.h"

namespace ibert {

struct RotaryArgs {
    const int8_t* qkv;
    const int16_t* table;
    const int32_t *positions, *slots;
    const int32_t* gamma[2];   // queries, keys
    int8_t *q, *k, *v;
    int64_t ld_qkv, ld_q, rows;
    int32_t wgs[3];            // workgroups of queries, of keys, of values
    int32_t teams[2];          // of a row's queries, and of its keys
    uint32_t teams_magic[2];
    int32_t heads_q, heads_kv, rot, max_pos, log_page, page_slots;
    int32_t shift[2];
    ibert_dyadic dy[2];
    int32_t fast[2];           // the dyadic's shift is 33 or more: the high half of one multiply-add, shifted
    int32_t v_l, v_r, v_m;     // DY(x) = ((x << v_l) * v_m + 2^(v_r + 31)) >> 32 >> v_r of a value
};

constexpr int RO_THREADS = 256, RO_TEAM_HEADS = 262144;

__device__ __forceinline__ int32_t byte_of(uint32_t p, int i) { return (int32_t)(int8_t)(p >> (8 * i)); }

// NH: heads of a row that a team of lanes takes one after the other.  With two the table's row, the row's slot and what else is the same for both is
// fetched once, and each lane finds the root and the reciprocal of one head for all; it halves the wavefronts, so it is for many rows.  us, one head /
// two, 32 + 8 heads of queries and keys of width 128: 1024 rows with norms 7.4 / 8.4, 2048 12.9 / 13.0, 4096 without 13.7 / 14.1, with 18.6 / 18.7, 6144 without 18.0 / 18.1, with
// 24.5 / 24.2, 8192 (the line, RO_TEAM_HEADS) without 27.7 / 25.8, with 37.2 / 35.1, 16384 without 56.2 / 49.2, with 70.3 / 62.8; 64 + 8 heads, 3072 rows without 15.3 / 15.9, 4096 (the line)
// 20.0 / 20.0, with 28.3 / 26.9.  As many keys as queries gain below the line too: 16 + 16 heads, 8192 rows without 34.0 / 29.0, with 40.5 / 35.8.
// (Four heads: 132 registers, 69.7 where two took 66.9.  Width 64, 2 lanes a head: no change at 16384 rows.)
template <int D, bool INTERLEAVED, int P, int NH>
__device__ __forceinline__ void rotate_heads(const RotaryArgs& a, int32_t wg, int kind)
{
    constexpr int LPH = D / (2 * P), W = P / 4;            // lanes of a head; dwords of a half
    static_assert(NH == 1 || (NH == 2 && LPH == 4), "heads of a team");
    typedef uint32_t words __attribute__((ext_vector_type(W)));
    const int heads = kind ? a.heads_kv : a.heads_q;
    const int32_t team = wg * (RO_THREADS / LPH) + threadIdx.x / LPH, row = udiv_fix(team, a.teams[kind], a.teams_magic[kind]);
    const int j = threadIdx.x % LPH;
    if (row >= (int32_t)a.rows) return;                    // (the lanes of a team together)
    const int head = (team - row * a.teams[kind]) * NH;
    const int32_t slot = a.slots[row];
    if ((uint32_t)slot >= (uint32_t)a.page_slots) return;
    const bool turned = 2 * P * j < a.rot;
    const int c0 = turned && !INTERLEAVED ? P * j : 2 * P * j, c1 = turned && !INTERLEAVED ? P * j + a.rot / 2 : 2 * P * j + P;
    const int8_t* src = a.qkv + row * a.ld_qkv + (kind ? a.heads_q : 0) * D;
    words w0[NH], w1[NH];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        const int8_t* from = src + (head + n < heads ? head + n : heads - 1) * D;
        w0[n] = *reinterpret_cast<const words*>(from + c0);
        w1[n] = *reinterpret_cast<const words*>(from + c1);
    }
    uint32_t cs[P];
    if (turned) {
        const int32_t pos = clamp_i32(a.positions[row], 0, a.max_pos - 1);
        const uint4* t = reinterpret_cast<const uint4*>(a.table + ((int64_t)pos * (a.rot / 2) + P * j) * 2);
#pragma unroll
        for (int i = 0; i < P / 4; ++i) {
            const uint4 w = t[i];
            cs[4 * i] = w.x; cs[4 * i + 1] = w.y; cs[4 * i + 2] = w.z; cs[4 * i + 3] = w.w;
        }
    }
    const int32_t* gamma = a.gamma[kind];
    int32_t f[NH];
    if (gamma) {
        int32_t mine = 0;
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            int32_t ss = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                ss = __builtin_amdgcn_sdot4((int32_t)w0[n][i], (int32_t)w0[n][i], ss, false);
                ss = __builtin_amdgcn_sdot4((int32_t)w1[n][i], (int32_t)w1[n][i], ss, false);
            }
            const auto add = [](int32_t p, int32_t q) { return p + q; };
            ss = add(ss, dpp_mov<0xB1>(ss));
            if (LPH > 2) ss = add(ss, dpp_mov<0x4E>(ss));
            if (LPH > 4) ss = add(ss, dpp_mov<0x141>(ss));
            mine = NH == 1 || n == (j & 1) ? ss : mine;
        }
        // sum <= 2^14 D: the mean's 16 fractional bits make it at most 2^30
        uint32_t sigma = isqrt_floor_lane((uint32_t)mine * (65536u / D));
        sigma = sigma < 1 ? 1 : sigma;
        const int32_t r = (int32_t)((1u << 30) / sigma);
        f[0] = r;
        if constexpr (NH == 2) {
            f[0] = dpp_mov<0x00>(r);                       // lane 0 of the team's, and lane 1's
            f[1] = dpp_mov<0x55>(r);
        }
    }
    const int32_t shift = a.shift[kind], norm_rnd = 1 << ((shift - 1) & 31);
    const ibert_dyadic dy = a.dy[kind];
    const int64_t rnd = (int64_t)1 << ((dy.s - 1) & 63);
    const int64_t page = slot >> a.log_page;
    const int t = slot & ((1 << a.log_page) - 1);
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        if (NH > 1 && head + n >= heads) return;
        int32_t x[2 * P];
#pragma unroll
        for (int i = 0; i < P; ++i) { x[i] = byte_of(w0[n][i / 4], i & 3); x[P + i] = byte_of(w1[n][i / 4], i & 3); }
        if (gamma) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int4* g4 = reinterpret_cast<const int4*>(gamma + (half ? c1 : c0));
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const int4 w = g4[i];
                    const int32_t gm[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        int32_t& u = x[P * half + 4 * i + r];
                        u = clamp_i32(smad24((u * f[n]) >> 12, gm[r], norm_rnd) >> shift, -32767, 32767);
                    }
                }
            }
        }
        if (turned) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int32_t c = (int32_t)(int16_t)cs[i], s = (int32_t)cs[i] >> 16;
                int32_t& p = x[INTERLEAVED ? 2 * i : i];
                int32_t& q = x[INTERLEAVED ? 2 * i + 1 : P + i];
                const int32_t y = smul24(p, c) - smul24(q, s);
                q = smad24(p, s, smul24(q, c));
                p = y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2 * P; ++i) x[i] <<= 14;
        }
        if (a.fast[kind]) {
#pragma unroll
            for (int i = 0; i < 2 * P; ++i) x[i] = med3_const<-127, 127>((int32_t)(((int64_t)x[i] * dy.m + rnd) >> 32) >> ((dy.s - 32) & 31));
        } else {
#pragma unroll
            for (int i = 0; i < 2 * P; ++i) x[i] = clamp_i64_to_i32(dyadic64(x[i], dy.m, dy.s), 127);
        }
        words o0, o1;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            o0[i] = pack4_perm(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
            o1[i] = pack4_perm(x[P + 4 * i], x[P + 4 * i + 1], x[P + 4 * i + 2], x[P + 4 * i + 3]);
        }
        if (kind == 0) {
            int8_t* dst = a.q + row * a.ld_q + (head + n) * D;
            *reinterpret_cast<words*>(dst + c0) = o0;
            *reinterpret_cast<words*>(dst + c1) = o1;
        } else {
            int8_t* dst = a.k + (((page * a.heads_kv + head + n) << a.log_page) + (t & ~15)) * D + (t & 15) * 16;
            *reinterpret_cast<words*>(dst + (c0 >> 4) * 256 + (c0 & 15)) = o0;
            *reinterpret_cast<words*>(dst + (c1 >> 4) * 256 + (c1 & 15)) = o1;
        }
    }
}

// 16 values of a row, requantized.
__device__ __forceinline__ void value_row(const RotaryArgs& a, const int8_t* src, uint32_t (&y)[4])
{
    const uint4 p = *reinterpret_cast<const uint4*>(src);
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
    const int64_t rnd = (int64_t)1 << (a.v_r + 31);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int32_t x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int32_t v = (int32_t)(((int64_t)(int32_t)((uint32_t)byte_of(w[i], r) << a.v_l) * a.v_m + rnd) >> 32) >> a.v_r;
            x[r] = med3_const<-127, 127>(v);
        }
        y[i] = pack4_perm(x[0], x[1], x[2], x[3]);
    }
}

template <int D>
__device__ __forceinline__ void append_values(const RotaryArgs& a, int32_t wg, uint32_t* lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int window = wg / a.heads_kv, head = wg - window * a.heads_kv;
    const int64_t row0 = (int64_t)window * 64, row = row0 + lane;
    // slots of the 64 rows, of those before and of those behind; which continue the row before
    const auto slot_at = [&](int64_t r) { return r >= 0 && r < a.rows ? a.slots[r] : -1; };
    const int32_t s0 = slot_at(row - 64), s1 = slot_at(row), s2 = slot_at(row + 64);
    const auto goes_on = [&](int32_t s, int32_t first_before) {
        const int32_t b = __shfl_up(s, 1), before = lane ? b : first_before;
        return __builtin_amdgcn_ballot_w64(s > 0 && (uint32_t)s < (uint32_t)a.page_slots && s == (int32_t)((uint32_t)before + 1u));
    };
    const uint64_t g0 = goes_on(s0, -1), g1 = goes_on(s1, __shfl(s0, 63)), g2 = goes_on(s2, __shfl(s1, 63));
    const bool in = (uint32_t)s1 < (uint32_t)a.page_slots;
    // The rows on the slots around this one that are in the same block of the cache: how many behind this row, how many before it.
    int after = 0, before = 0;
    if (in) {
        uint64_t run = g2;                                 // bit k: row lane + 1 + k goes on from the one before it
        if (lane < 63) run = (g1 >> (lane + 1)) | (g2 << (63 - lane));
        after = __builtin_ctzll(~run | (uint64_t)1 << 63);
        run = lane < 63 ? (g1 << (63 - lane)) | (g0 >> (lane + 1)) : g1;        // from bit 63 down: row lane and those before it
        before = __builtin_clzll(~run | 1);
        after = after < 63 - (s1 & 63) ? after : 63 - (s1 & 63);
        before = before < (s1 & 63) ? before : s1 & 63;
    }
    const bool alone = in && after + before < 3;           // (fewer than four rows: each by itself)
    uint64_t starts = __builtin_amdgcn_ballot_w64(in && !alone && before == 0);
    uint32_t* const mine = lds + wave * 256;
    for (int j = wave; j < D / 16; j += RO_THREADS / 64) {
        const int8_t* src = a.qkv + (a.heads_q + a.heads_kv + head) * D + 16 * j;
        if (alone) {
            uint32_t y[4];
            value_row(a, src + row * a.ld_qkv, y);
            const int64_t page = s1 >> a.log_page;
            const int t = s1 & ((1 << a.log_page) - 1);
            int8_t* dst = a.v + (((page * a.heads_kv + head) << a.log_page) + (t & ~63)) * D + j * 1024 + ((t >> 2) & 3) * 256 + ((t >> 4) & 3) * 4 + (t & 3);
#pragma unroll
            for (int i = 0; i < 16; ++i) dst[16 * i] = (int8_t)byte_of(y[i / 4], i & 3);
        }
        for (uint64_t left = starts; left; left &= left - 1) {
            // lane = token of the block; rows `first` .. on tokens from .. to - 1
            const int first = __builtin_ctzll(left);
            const int32_t slot = __builtin_amdgcn_readlane(s1, first), from = slot & 63, to = from + 1 + __builtin_amdgcn_readlane(after, first);
            uint32_t y[4] = {0, 0, 0, 0};
            if (lane >= from && lane < to) value_row(a, src + (row0 + first + lane - from) * a.ld_qkv, y);
            // four rows are four neighbouring lanes: byte r' of lane r becomes byte r of lane r'
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t o = (uint32_t)dpp_mov<0xB1>((int32_t)y[i]);
                y[i] = __builtin_amdgcn_perm(o, y[i], lane & 1 ? 0x03070105u : 0x06020400u);
                const uint32_t q = (uint32_t)dpp_mov<0x4E>((int32_t)y[i]);
                y[i] = __builtin_amdgcn_perm(q, y[i], lane & 2 ? 0x03020706u : 0x05040100u);
            }
            // lane 16 i + 4 g + r: its dword of channel 4 n + r goes to [g][channel][i]
#pragma unroll
            for (int n = 0; n < 4; ++n) mine[((lane >> 2) & 3) * 64 + (4 * n + (lane & 3)) * 4 + (lane >> 4)] = y[n];
            __builtin_amdgcn_wave_barrier();
            const uint4 o = *reinterpret_cast<const uint4*>(mine + 4 * lane);
            __builtin_amdgcn_wave_barrier();
            const int64_t page = slot >> a.log_page;
            const int t = slot & ((1 << a.log_page) - 1) & ~63;
            int8_t* dst = a.v + (((page * a.heads_kv + head) << a.log_page) + t) * D + j * 1024 + lane * 16;
            if (to - from == 64) {
                *reinterpret_cast<uint4*>(dst) = o;
            } else {
                const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = 16 * i + 4 * (lane >> 4);
                    if (token >= from && token + 4 <= to) {
                        *reinterpret_cast<uint32_t*>(dst + 4 * i) = w[i];
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (token + r >= from && token + r < to) dst[4 * i + r] = (int8_t)byte_of(w[i], r);
                    }
                }
            }
        }
    }
}

template <int D, bool INTERLEAVED, int P, int NH>
__global__ __launch_bounds__(RO_THREADS) void rotary_append_kernel(RotaryArgs a)
{
    __shared__ __attribute__((aligned(16))) uint32_t lds[RO_THREADS / 64 * 256];
    const int32_t wg = (int32_t)blockIdx.x;
    // (values first: theirs is the longest chain of loads)
    if (wg < a.wgs[2]) append_values<D>(a, wg, lds);
    else if (wg < a.wgs[2] + a.wgs[1]) rotate_heads<D, INTERLEAVED, P, NH>(a, wg - a.wgs[2], 1);
    else rotate_heads<D, INTERLEAVED, P, NH>(a, wg - a.wgs[2] - a.wgs[1], 0);
}

// The same multiplier with a shift of at least `least`, where 31 bits hold it: DY(x; 2m, s + 1) = DY(x; m, s).
static ibert_dyadic shifted(ibert_dyadic d, int least)
{
    while (d.s < least && d.m < (1 << 30) && d.m > -(1 << 30)) { d.m *= 2; ++d.s; }
    return d;
}

template <int D, bool INTERLEAVED, int P, int NH>
static int launch_rotary(RotaryArgs& a, hipStream_t stream)
{
    constexpr int per = RO_THREADS / (D / (2 * P));
    const int32_t heads[2] = {a.heads_q, a.heads_kv};
    for (int k = 0; k < 2; ++k) {
        a.teams[k] = (heads[k] + NH - 1) / NH;
        a.teams_magic[k] = udiv_magic(a.teams[k]);
        a.wgs[k] = (int32_t)((a.rows * a.teams[k] + per - 1) / per);
    }
    a.wgs[2] = (int32_t)((a.rows + 63) / 64 * a.heads_kv);
    hipLaunchKernelGGL((rotary_append_kernel<D, INTERLEAVED, P, NH>), dim3((unsigned)(a.wgs[0] + a.wgs[1] + a.wgs[2])), dim3(RO_THREADS), 0, stream, a);
    IBERT_LAUNCH_CHECK("rotary_append_kernel");
    static const KernelName name("rotary_append_kernel<%d, %s, %d, %d>", D, INTERLEAVED ? "true" : "false", P, NH);
    g_last_kernel = name.text;
    return IBERT_OK;
}

static int g_rotary_heads = -1;         // see ibert_rotary_override

template <int D>
static int launch_rotary(RotaryArgs& a, bool interleaved, hipStream_t stream)
{
    if (a.rot % 32) return interleaved ? launch_rotary<D, true, 8, 1>(a, stream) : launch_rotary<D, false, 8, 1>(a, stream);
    if constexpr (D == 128) {
        if (g_rotary_heads < 0 ? a.rows * a.heads_q >= RO_TEAM_HEADS : g_rotary_heads == 2) return interleaved ? launch_rotary<D, true, 16, 2>(a, stream) : launch_rotary<D, false, 16, 2>(a, stream);
    }
    return interleaved ? launch_rotary<D, true, 16, 1>(a, stream) : launch_rotary<D, false, 16, 1>(a, stream);
}

}  // namespace ibert

extern "C" void ibert_rotary_override(int32_t heads) { ibert::g_rotary_heads = heads; }

extern "C" int ibert_rotary_append_i(const ibert_rotary_desc* desc, const ibert_kv_cache* cache, const int8_t* qkv, int64_t ld_qkv,
                                     const int16_t* table, const int32_t* positions, const int32_t* slots, const int32_t* q_gamma,
                                     const int32_t* k_gamma, int64_t rows, int8_t* q, int64_t ld_q, void* stream)
{
    using namespace ibert;
    if (!desc || !cache) return IBERT_ERR_NULL;
    if (const int rc = check_cache(cache)) return rc;
    const ibert_rotary_desc& d = *desc;
    const int D = cache->head_dim;
    if (rows < 0 || d.heads_q < 1 || d.heads_q > (1 << 20) || d.heads_q % cache->heads_kv) return IBERT_ERR_SHAPE;
    const int32_t heads = d.heads_q + 2 * cache->heads_kv;
    if (ld_qkv < (int64_t)heads * D || ld_q < (int64_t)d.heads_q * D) return IBERT_ERR_SHAPE;
    if (d.rot_dim < 0 || d.rot_dim > D || d.rot_dim % 16 || (d.layout != IBERT_ROTARY_HALF && d.layout != IBERT_ROTARY_INTERLEAVED) ||
        !dyadic_ok(d.q_dy) || !dyadic_ok(d.k_dy) || !dyadic_ok(d.v_dy) || (d.rot_dim > 0 && d.max_pos < 1) ||
        (q_gamma && (d.q_norm_shift < 1 || d.q_norm_shift > 30)) || (k_gamma && (d.k_norm_shift < 1 || d.k_norm_shift > 30))) return IBERT_ERR_PARAM_RANGE;
    if (rows == 0) return IBERT_OK;
    if (rows > INT32_MAX / heads - 256) return IBERT_ERR_SHAPE;          // (teams of lanes are counted in 32 bits)
    if (!qkv || !slots || !q || !cache->k || !cache->v || (d.rot_dim > 0 && (!table || !positions))) return IBERT_ERR_NULL;
    if (!aligned(qkv, 16) || !aligned(q, 16) || !aligned(cache->k, 16) || !aligned(cache->v, 16) || !aligned(table, 16) || ld_qkv % 16 || ld_q % 16 ||
        !aligned(q_gamma, 16) || !aligned(k_gamma, 16)) return IBERT_ERR_ALIGN;
    RotaryArgs a;
    a.qkv = qkv; a.table = table; a.positions = positions; a.slots = slots; a.gamma[0] = q_gamma; a.gamma[1] = k_gamma;
    a.q = q; a.k = cache->k; a.v = cache->v; a.ld_qkv = ld_qkv; a.ld_q = ld_q; a.rows = rows;
    a.heads_q = d.heads_q; a.heads_kv = cache->heads_kv; a.rot = d.rot_dim; a.max_pos = d.max_pos;
    a.log_page = __builtin_ctz((unsigned)cache->page_size); a.page_slots = cache->num_pages * cache->page_size;
    a.shift[0] = d.q_norm_shift; a.shift[1] = d.k_norm_shift; 
    a.dy[0] = shifted(d.q_dy, 33); a.dy[1] = shifted(d.k_dy, 33);
    a.fast[0] = a.dy[0].s >= 33; a.fast[1] = a.dy[1].s >= 33;
    // (a shift that stays below 9 stands for a multiplier of 2^21 and more: any value but 0 comes out at the end of the range)
    ibert_dyadic v = shifted(d.v_dy, 33);
    if (v.s < 9) v.s = 9;
    a.v_m = v.m; a.v_l = v.s < 33 ? 33 - v.s : 0; a.v_r = v.s < 33 ? 1 : v.s - 32;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return D == 64 ? launch_rotary<64>(a, d.layout == IBERT_ROTARY_INTERLEAVED, st) : launch_rotary<128>(a, d.layout == IBERT_ROTARY_INTERLEAVED, st);
}
