// Rotary positions of queries and keys, the optional norm of each head in front of them, and the append of keys and values to
// the paged cache (ibert_rotary_append_i): one pass over the packed QKV rows.
//
// A head takes D / 16 lanes, 16 channels each, as two pieces of 8: the two halves of 8 pairs, so that no value crosses lanes
// for the rotation.  (Half layout: channels 8 j .. and 8 j + R/2 ..; interleaved, and behind the rotated part: 16 j .. and
// 16 j + 8 ..)  The norm adds up squares over the head's lanes in registers.  Cosine and sine stand in a table with 14
// fractional bits: a rotated value is below 2^30, and its requantization is the same 64-bit step as a MatMul's.
// Bound: HBM and the memory pipeline (16 bytes in and out of a lane).
#include "layernorm_math.h"

namespace ibert {

struct RotaryArgs {
    const int8_t* qkv;
    const int16_t* table;
    const int32_t *positions, *slots, *q_gamma, *k_gamma;
    int8_t *q, *k, *v;
    int64_t ld_qkv, ld_q;
    int64_t groups;            // rows * heads of all three kinds
    int32_t heads, heads_q, heads_kv, rot, max_pos, log_page, page_slots;
    int32_t q_shift, k_shift;
    ibert_dyadic q_dy, k_dy, v_dy;
};

constexpr int RO_THREADS = 256;

// DY(x; m, s), clamped to 8 bits.
__device__ __forceinline__ int32_t requant8(int32_t x, ibert_dyadic dy)
{
    return clamp_i64_to_i32(dyadic64(x, dy.m, dy.s), 127);
}

__device__ __forceinline__ void unpack8(uint2 p, int32_t* x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (int32_t)(int8_t)((i < 4 ? p.x : p.y) >> (8 * (i & 3)));
}
__device__ __forceinline__ uint2 pack8(const int32_t* x)
{
    return make_uint2(pack4_perm(x[0], x[1], x[2], x[3]), pack4_perm(x[4], x[5], x[6], x[7]));
}

template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(RO_THREADS) void rotary_append_kernel(RotaryArgs a)
{
    constexpr int LPH = D / 16;
    const int64_t group = (int64_t)blockIdx.x * (RO_THREADS / LPH) + threadIdx.x / LPH;
    if (group >= a.groups) return;                         // (the lanes of a head together)
    const int j = threadIdx.x % LPH;
    const int64_t row = group / a.heads;
    const int head = (int)(group - row * a.heads);
    const int32_t slot = a.slots[row];
    if ((uint32_t)slot >= (uint32_t)a.page_slots) return;
    const int8_t* src = a.qkv + row * a.ld_qkv + head * D;
    const int kv = head - a.heads_q;                       // which key head, or heads_kv + which value head
    const int64_t page = slot >> a.log_page;
    const int t = slot & ((1 << a.log_page) - 1);

    if (kv >= a.heads_kv) {
        int32_t x[16];
        const uint4 p = *reinterpret_cast<const uint4*>(src + 16 * j);
        unpack8(make_uint2(p.x, p.y), x);
        unpack8(make_uint2(p.z, p.w), x + 8);
        int8_t* dst = a.v + (((page * a.heads_kv + (kv - a.heads_kv)) << a.log_page) + (t & ~63)) * D + j * 1024 + ((t >> 2) & 3) * 256 +
                      ((t >> 4) & 3) * 4 + (t & 3);
#pragma unroll
        for (int i = 0; i < 16; ++i) dst[16 * i] = (int8_t)requant8(x[i], a.v_dy);
        return;
    }
    const bool turned = 16 * j < a.rot;
    const int c0 = turned && !INTERLEAVED ? 8 * j : 16 * j, c1 = turned && !INTERLEAVED ? 8 * j + a.rot / 2 : 16 * j + 8;
    int32_t x[16];
    unpack8(*reinterpret_cast<const uint2*>(src + c0), x);
    unpack8(*reinterpret_cast<const uint2*>(src + c1), x + 8);

    const int32_t* gamma = kv < 0 ? a.q_gamma : a.k_gamma;
    if (gamma) {
        const int32_t shift = kv < 0 ? a.q_shift : a.k_shift;
        int32_t ss = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss += smul24(x[i], x[i]);
        const auto add = [](int32_t p, int32_t q) { return p + q; };
        ss = add(ss, dpp_mov<0xB1>(ss));
        ss = add(ss, dpp_mov<0x4E>(ss));
        if (LPH > 4) ss = add(ss, dpp_mov<0x141>(ss));
        // sum <= 2^14 D: the mean's 16 fractional bits make it less than 2^31
        uint32_t sigma = isqrt_floor_lane((uint32_t)ss * (65536u / D));
        sigma = sigma < 1 ? 1 : sigma;
        const int32_t f = (int32_t)((1u << 30) / sigma);
        const int32_t rnd = 1 << (shift - 1);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int32_t n = (x[i] * f) >> 12;
            x[i] = clamp_i32((n * gamma[i < 8 ? c0 + i : c1 + i - 8] + rnd) >> shift, -32767, 32767);
        }
    }
    if (turned) {
        int32_t pos = a.positions[row];
        pos = clamp_i32(pos, 0, a.max_pos - 1);
        const uint4* cs4 = reinterpret_cast<const uint4*>(a.table + ((int64_t)pos * (a.rot / 2) + 8 * j) * 2);
        const uint4 w0 = cs4[0], w1 = cs4[1];
        const uint32_t cs[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int32_t c = (int32_t)(int16_t)cs[i], s = (int32_t)cs[i] >> 16;
            int32_t& p = INTERLEAVED ? x[2 * i] : x[i];
            int32_t& q = INTERLEAVED ? x[2 * i + 1] : x[8 + i];
            const int32_t y = smul24(p, c) - smul24(q, s);
            q = smul24(p, s) + smul24(q, c);
            p = y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] <<= 14;
    }
    const ibert_dyadic dy = kv < 0 ? a.q_dy : a.k_dy;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = requant8(x[i], dy);
    if (kv < 0) {
        int8_t* dst = a.q + row * a.ld_q + head * D;
        *reinterpret_cast<uint2*>(dst + c0) = pack8(x);
        *reinterpret_cast<uint2*>(dst + c1) = pack8(x + 8);
    } else {
        int8_t* dst = a.k + (((page * a.heads_kv + kv) << a.log_page) + (t & ~15)) * D + (t & 15) * 16;
        *reinterpret_cast<uint2*>(dst + (c0 >> 4) * 256 + (c0 & 15)) = pack8(x);
        *reinterpret_cast<uint2*>(dst + (c1 >> 4) * 256 + (c1 & 15)) = pack8(x + 8);
    }
}

template <int D, bool INTERLEAVED>
static int launch_rotary(const RotaryArgs& a, hipStream_t stream)
{
    constexpr int per = RO_THREADS / (D / 16);
    const int64_t wgs = (a.groups + per - 1) / per;
    if (wgs > 0x7fffffffLL) return IBERT_ERR_SHAPE;
    hipLaunchKernelGGL((rotary_append_kernel<D, INTERLEAVED>), dim3((unsigned)wgs), dim3(RO_THREADS), 0, stream, a);
    IBERT_LAUNCH_CHECK("rotary_append_kernel");
    g_last_kernel = "rotary_append_kernel";
    return IBERT_OK;
}

}  // namespace ibert

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
    if (rows > INT64_MAX / heads) return IBERT_ERR_SHAPE;
    if (!qkv || !slots || !q || !cache->k || !cache->v || (d.rot_dim > 0 && (!table || !positions))) return IBERT_ERR_NULL;
    if (!aligned(qkv, 16) || !aligned(q, 16) || !aligned(cache->k, 16) || !aligned(cache->v, 16) || !aligned(table, 16) || ld_qkv % 16 || ld_q % 16)
        return IBERT_ERR_ALIGN;
    RotaryArgs a;
    a.qkv = qkv; a.table = table; a.positions = positions; a.slots = slots; a.q_gamma = q_gamma; a.k_gamma = k_gamma;
    a.q = q; a.k = cache->k; a.v = cache->v; a.ld_qkv = ld_qkv; a.ld_q = ld_q;
    a.groups = rows * heads; a.heads = heads; a.heads_q = d.heads_q; a.heads_kv = cache->heads_kv;
    a.rot = d.rot_dim; a.max_pos = d.max_pos;
    a.log_page = __builtin_ctz((unsigned)cache->page_size); a.page_slots = cache->num_pages * cache->page_size;
    a.q_shift = d.q_norm_shift; a.k_shift = d.k_norm_shift; a.q_dy = d.q_dy; a.k_dy = d.k_dy; a.v_dy = d.v_dy;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (d.layout == IBERT_ROTARY_INTERLEAVED) return D == 64 ? launch_rotary<64, true>(a, st) : launch_rotary<128, true>(a, st);
    return D == 64 ? launch_rotary<64, false>(a, st) : launch_rotary<128, false>(a, st);
}
