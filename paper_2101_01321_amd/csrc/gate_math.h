// The gated product of a feed-forward block on its two sums: activation of the gate (SiLU by the i-exp of Alg. 3, or the
// integer GELU of Alg. 2), times the up projection, requantized once.  Shared by every kernel that ends in it.
#pragma once
#include "common.h"
#include "gelu_math.h"

namespace ibert {

struct GateConst {
    int32_t silu;          // 1: SiLU, 0: GELU (its output requantization goes to 16 bits here)
    GeluConst gelu;
    int32_t m, s;          // requantization of the product
};

constexpr int32_t SIG_TOP = 124 * 124 + 8180;      // i-exp at 0 with the constants of Eq. 13 at S = ln2/64
constexpr int SIG_STEPS = 1024;                    // from 16 octaves on the sigmoid is one

// DY(x; m, s) without a case for s = 0, and a 64-bit value inside INT32 (the low half where the high one is its sign) or inside +-lim of it.
__device__ __forceinline__ int64_t dy64(int32_t x, int32_t m, int32_t s) { return ((int64_t)x * m + (((int64_t)1 << s) >> 1)) >> s; }
__device__ __forceinline__ int32_t into_32(int64_t v)
{
    const int32_t lo = (int32_t)v, hi = (int32_t)(v >> 32);
    return hi == lo >> 31 ? lo : (hi >> 31) ^ INT32_MAX;
}
__device__ __forceinline__ int32_t into(int64_t v, int32_t lim) { return med3_i32(into_32(v), -lim, lim); }

// Sigmoid of a distance d in [0, 1024] steps of ln2/64, 15 bits: TOP / (TOP + e) rounded to nearest.  The numerator stays below 2^30.
__host__ __device__ __forceinline__ uint32_t sigmoid15(uint32_t d)
{
    const uint32_t z = d >> 6, f = d & 63u, b = 124u - f;
    const uint32_t e = z < 16u ? (b * b + 8180u + ((1u << z) >> 1)) >> z : 0u;
    const uint32_t n = (uint32_t)SIG_TOP + e;
    return (((uint32_t)SIG_TOP << 15) + (n >> 1)) / n;
}

// SiLU of a gate on the scale ln2/1024, on the same scale.  |g| <= 65535 and p <= 2^15 keep the product and its rounding inside 32 bits.
__device__ __forceinline__ int32_t silu_of(int32_t g, uint32_t p)
{
    const int32_t q = g < 0 ? 32768 - (int32_t)p : (int32_t)p;
    return (g * q + 16384) >> 15;
}
__device__ __forceinline__ uint32_t silu_step(int32_t g)
{
    const uint32_t d = ((uint32_t)(g < 0 ? -g : g) + 8u) >> 4;
    return d < (uint32_t)SIG_STEPS ? d : (uint32_t)SIG_STEPS;
}

// As gelu_one, to 16 bits.
__device__ __forceinline__ int32_t gelu16(int32_t q, const GeluConst& a)
{
    int32_t u = q < 0 ? -q : q;
    u = u > -a.q_b ? -a.q_b : u;
    const int32_t v = u + a.q_b;
    const uint32_t poly = (uint32_t)v * (uint32_t)v + (uint32_t)a.q_c;
    const uint32_t erf = q < 0 ? 0u - poly : (q == 0 ? 0u : poly);
    const int32_t t = (int32_t)((uint32_t)q * (erf + (uint32_t)a.q_1));
    return into(dy64(t, a.m, a.s), 32767);
}

// The INT8 result of one pair of sums.
__device__ __forceinline__ int32_t gate_one(int32_t acc_g, int32_t acc_u, int32_t mg, int32_t sg, int32_t mu, int32_t su, const GateConst& c)
{
    const int32_t g = into(dy64(acc_g, mg, sg), c.silu ? 65535 : c.gelu.q_max);
    const int32_t u = into(dy64(acc_u, mu, su), 32767);
    const int32_t a = c.silu ? silu_of(g, sigmoid15(silu_step(g))) : gelu16(g, c.gelu);
    return into(dy64(a * u, c.m, c.s), 127);      // (65535 * 32767 < 2^31)
}

inline GateConst gate_const(const ibert_gate_params& p)
{
    GateConst c{};
    c.silu = p.activation == IBERT_GATE_SILU;
    if (!c.silu) c.gelu = GeluConst{p.gelu.q_b, p.gelu.q_c, p.gelu.q_1, p.gelu.q_max, p.gelu.out.m, p.gelu.out.s};
    c.m = p.out_dy.m;
    c.s = p.out_dy.s;
    return c;
}

}  // namespace ibert
