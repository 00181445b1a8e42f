// How a product of few rows is laid out (RowsPlan), and its launch.  One unit per group size instantiates launch_rows.
#pragma once
#include "rows_kernel.h"

namespace ibert {

// ring: rows_ring_kernel, else rows_any_kernel.  A workgroup takes 8 br rows and nt tiles of 16 channels (of a gated block nt pairs).
struct RowsPlan {
    int32_t br, nt, ring;
};

template <bool W4, int G>
int launch_rows(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream);

constexpr int ROWS_LDS = 163840;

// Launches workgroups of tm rows by tn channels, those of the same channels on the same XCD; in pieces of rows where there would be 2^32 threads.
template <typename F, typename Name>
int rows_pieces(F kern, RowsArgs g, int tm, int tn, size_t lds, hipStream_t stream, Name name)
{
    const int64_t M = g.M, across = ((int64_t)g.N + tn - 1) / tn, across8 = (across + 7) / 8 * 8, down = (M + tm - 1) / tm;
    const int64_t most = (1 << 22) / across8;                       // (N is at most 2^24, across8 2^20)
    const int8_t *A = g.A, *R = g.R;
    char* C = static_cast<char*>(g.C);
    const int64_t elem = g.out_dtype == IBERT_I8 ? 1 : (g.out_dtype == IBERT_I16 ? 2 : 4);
    for (int64_t d0 = 0; d0 < down; d0 += most) {
        const int64_t m0 = d0 * tm, n = down - d0 < most ? down - d0 : most;
        g.A = A + m0 * g.lda;
        g.R = R ? R + m0 * g.ldr : nullptr;
        g.C = C + m0 * g.ldc * elem;
        g.M = (int32_t)(M - m0 < n * tm ? M - m0 : n * tm);
        g.down = (int32_t)n;
        g.down_magic = udiv_magic(g.down);
        g.across = (int32_t)across;
        hipLaunchKernelGGL(kern, dim3((unsigned)(across8 * n)), dim3(ROWS_THREADS), lds, stream, g);
        IBERT_LAUNCH_CHECK("rows_kernel");
    }
    g_last_kernel = name();
    return IBERT_OK;
}

// Can rows_ring_kernel serve these operands, and with how many stages (0: it cannot)?  As many as there is use for, at most four, of what LDS holds beside two
// more workgroups where there are that many for a unit: us, [1,4096] x 12288 pairs of 4 bits, 768 workgroups, with one stage 13.3, two (three workgroups) 12.3, three
// (two workgroups) 13.2, four (one) 19.8.
inline int ring_stages(const RowsArgs& g, bool w4, int br, int tiles, bool gated, int group, bool zeros, size_t* lds)
{
    const int tn = 16 * (gated ? tiles / 2 : tiles);
    if (!g.a_vec || g.lda > (1 << 24) || (w4 ? g.per > 32 : !g.w_vec)) return 0;
    const size_t sc = w4 ? (size_t)((g.per * 16 * (128 / group) + 255) & ~255) * tiles * (zeros ? 2 : 1) : 0, sums = (size_t)32 * br * (16 * tiles + 4);
    const size_t stage = (size_t)(br + tiles * (w4 ? 1 : 2)) * 1024;
    auto bytes = [&](int n) { return 8 * (sc + (n * stage > sums ? n * stage : sums)); };
    const int64_t blocks = (((int64_t)g.N + tn - 1) / tn) * (((int64_t)g.M + 8 * br - 1) / (8 * br));
    const size_t side = blocks <= 256 ? 1 : (blocks <= 512 ? 2 : 3);
    int n = g.per < 4 ? g.per : 4;
    while (n > 1 && bytes(n) > ROWS_LDS / side) --n;
    *lds = bytes(n);
    return *lds <= (size_t)ROWS_LDS ? n : 0;
}

template <bool W4, int BR, int NT, int G, bool ZERO, bool GATED>
int launch_ring_as(RowsArgs g, hipStream_t stream)
{
    auto kern = rows_ring_kernel<W4, BR, NT, G, ZERO, GATED>;
    static bool attr_done = false;
    if (!attr_done) {
        IBERT_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, ROWS_LDS));
        attr_done = true;
    }
    constexpr int NH = GATED ? NT / 2 : NT, TM = 8 * BR;
    size_t lds;
    g.stages = ring_stages(g, W4, BR, NT, GATED, G, ZERO, &lds);
    if (g.stages == 0) return IBERT_ERR_NOT_IMPLEMENTED;
    return rows_pieces(kern, g, TM, 16 * NH, lds, stream, [] {
        static const KernelName name("rows_ring_kernel<%s, %d, %d, %d, %s, %s>", W4 ? "true" : "false", BR, NT, G, ZERO ? "true" : "false", GATED ? "true" : "false");
        return name.text;
    });
}

// The tiles that plan_ring picks, and those that it makes smaller where LDS is short: one tile (pair) of channels by up to four blocks of rows; beside them eight blocks by two
// pairs of INT8 weights, four blocks by two pairs of 4-bit ones, and up to four blocks by two tiles, or four by four, of a product alone.
template <bool W4, int G, bool ZERO, bool GATED>
int launch_ring(const RowsArgs& g, const RowsPlan& plan, hipStream_t stream)
{
    constexpr int PER = GATED ? 2 : 1;
    if (plan.nt == 1) {
        if (plan.br == 1) return launch_ring_as<W4, 1, PER, G, ZERO, GATED>(g, stream);
        if (plan.br == 2) return launch_ring_as<W4, 2, PER, G, ZERO, GATED>(g, stream);
        return launch_ring_as<W4, 4, PER, G, ZERO, GATED>(g, stream);
    }
    if constexpr (GATED) return launch_ring_as<W4, W4 ? 4 : 8, 4, G, ZERO, GATED>(g, stream);
    else {
        if (plan.nt == 4) return launch_ring_as<W4, 4, 4, G, ZERO, GATED>(g, stream);
        if (plan.br == 1) return launch_ring_as<W4, 1, 2, G, ZERO, GATED>(g, stream);
        if (plan.br == 2) return launch_ring_as<W4, 2, 2, G, ZERO, GATED>(g, stream);
        return launch_ring_as<W4, 4, 2, G, ZERO, GATED>(g, stream);
    }
}

template <bool W4, int BR, int NT, int G, bool ZERO, bool GATED>
int launch_any_as(RowsArgs g, hipStream_t stream)
{
    auto kern = rows_any_kernel<W4, BR, NT, G, ZERO, GATED>;
    static bool attr_done = false;
    if (!attr_done) {
        IBERT_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, ROWS_LDS));
        attr_done = true;
    }
    constexpr int STAGE = (BR + (W4 ? 0 : 2 * NT)) * 1024, SUMS = 8 * BR * (16 * NT + 4) * (W4 ? 8 : 4);
    constexpr int OWN = W4 ? STAGE + SUMS : (STAGE > SUMS ? STAGE : SUMS);
    static_assert(8 * OWN <= ROWS_LDS, "LDS of a workgroup");
    return rows_pieces(kern, g, 8 * BR, 16 * (GATED ? NT / 2 : NT), 8 * OWN, stream, [] {
        static const KernelName name("rows_any_kernel<%s, %d, %d, %d, %s, %s>", W4 ? "true" : "false", BR, NT, G, ZERO ? "true" : "false", GATED ? "true" : "false");
        return name.text;
    });
}

// (One or four blocks of rows; by two pairs of INT8 tiles and four or eight blocks [1000,2001] x 4000 takes 177 us, by one 155, [2711,579] x 704 54 and 48 / 42.)
template <bool W4, int G, bool ZERO, bool GATED>
int launch_any(const RowsArgs& g, const RowsPlan& plan, hipStream_t stream)
{
    if (plan.br >= 2) return launch_any_as<W4, 4, 2, G, ZERO, GATED>(g, stream);
    if constexpr (W4 && !GATED) if (plan.nt == 1) return launch_any_as<W4, 1, 1, G, ZERO, GATED>(g, stream);
    return launch_any_as<W4, 1, 2, G, ZERO, GATED>(g, stream);
}

#define IBERT_ROWS_UNIT(W4_, G_)                                                                                          \
    template <>                                                                                                           \
    int launch_rows<W4_, G_>(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream)                \
    {                                                                                                                     \
        if constexpr (W4_) {                                                                                              \
            if (gated) {                                                                                                  \
                if (plan.ring) return zeros ? launch_ring<W4_, G_, true, true>(g, plan, stream) : launch_ring<W4_, G_, false, true>(g, plan, stream);     \
                return zeros ? launch_any<W4_, G_, true, true>(g, plan, stream) : launch_any<W4_, G_, false, true>(g, plan, stream);                      \
            }                                                                                                             \
            if (plan.ring) return zeros ? launch_ring<W4_, G_, true, false>(g, plan, stream) : launch_ring<W4_, G_, false, false>(g, plan, stream);       \
            return zeros ? launch_any<W4_, G_, true, false>(g, plan, stream) : launch_any<W4_, G_, false, false>(g, plan, stream);                        \
        } else return plan.ring ? launch_ring<W4_, G_, false, true>(g, plan, stream) : launch_any<W4_, G_, false, true>(g, plan, stream);                 \
    }

}  // namespace ibert
