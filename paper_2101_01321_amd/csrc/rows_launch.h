// How a product of few rows is laid out (RowsPlan), and its launch.  One unit per group size instantiates launch_rows.
#pragma once
#include "rows_kernel.h"

namespace ibert {

// ring: rows_ring_kernel, whose workgroups take 8 br rows (br: 1, 2, 4, 8) and nt tiles of channels.  Else rows of a workgroup / 16 (1, 2, 4); tiles of 16 channels to a wavefront, of each matrix of a gated block (1, 2); log2 of its groups of channels
struct RowsPlan {
    int32_t mt, nt, cg, ring, br;
};

template <bool W4, int G>
int launch_rows(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream);

constexpr int ROWS_LDS = 163840;

// Launches workgroups of tm rows by tn channels, those of the same channels on the same XCD; in pieces of rows where there would be 2^32 threads.
template <typename F, typename Name>
int rows_pieces(F kern, RowsArgs g, int tm, int tn, size_t lds, hipStream_t stream, Name name)
{
    const int64_t M = g.M, across = ((int64_t)g.N + tn - 1) / tn, down = (M + tm - 1) / tm, most = (1 << 22) / across < 1 ? 1 : (1 << 22) / across;
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
        g.across = (int32_t)across;
        hipLaunchKernelGGL(kern, dim3((unsigned)((across + 7) / 8 * 8 * n)), dim3(ROWS_THREADS), lds, stream, g);
        IBERT_LAUNCH_CHECK("rows_kernel");
    }
    g_last_kernel = name();
    return IBERT_OK;
}

template <bool W4, int MT, int NT, int G, bool ZERO, bool GATED>
int launch_rows_as(RowsArgs g, const RowsPlan& plan, hipStream_t stream)
{
    auto kern = rows_kernel<W4, MT, NT, G, ZERO, GATED>;
    static bool attr_done = false;
    if (!attr_done) {
        IBERT_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, ROWS_LDS));
        attr_done = true;
    }
    constexpr int NH = GATED ? NT / 2 : NT;
    const int32_t rows = g.M < 16 * MT ? g.M : 16 * MT;
    g.mp = 0;
    while ((1 << g.mp) < rows) ++g.mp;
    g.cg = plan.cg;
    g.chunks = (g.K + 127) / 128;
    // a slab: all of K where 64 KB (or what the sums leave) hold it, else whole rounds of the wavefronts' rings; fewer groups of channels where not one round fits
    auto sums = [&]() { return (int64_t)16 * MT * (16 * NT << g.cg) * (W4 ? 8 : 4); };
    auto round = [&]() { return (8 >> g.cg) * rows_ring(MT); };
    while (g.cg > 0 && sums() + ((int64_t)round() << 7 << g.mp) > ROWS_LDS) --g.cg;
    const int64_t left = ROWS_LDS - sums(), room = left < 65536 ? left : 65536;
    const int32_t most = (int32_t)(room >> 7 >> g.mp) / round() * round();
    g.slab = (g.chunks + round() - 1) / round() * round();
    if (g.slab > most) g.slab = most < round() ? round() : most;
    const size_t lds = ((size_t)g.slab << 7 << g.mp) + (size_t)sums();
    if (lds > (size_t)ROWS_LDS) return IBERT_ERR_NOT_IMPLEMENTED;
    return rows_pieces(kern, g, 16 * MT, 16 * NH << g.cg, lds, stream, [] {
        static const KernelName name("rows_kernel<%s, %d, %d, %d, %s, %s>", W4 ? "true" : "false", MT, NT, G, ZERO ? "true" : "false", GATED ? "true" : "false");
        return name.text;
    });
}

// Can rows_ring_kernel serve these operands, and with how many stages (0: it cannot)?  As many as there is use for, at most four, of what LDS holds beside two
// more workgroups where there are that many for a unit: us, [1,4096] x 12288 pairs of 4 bits, 768 workgroups, with one stage 13.3, two (three workgroups) 12.3, three
// (two workgroups) 13.2, four (one) 19.8.
inline int ring_stages(const RowsArgs& g, bool w4, int br, int tiles, bool gated, int group, bool zeros, int* per, size_t* lds)
{
    const int chunks = (g.K + 127) / 128, tn = 16 * (gated ? tiles / 2 : tiles);
    *per = (chunks + 7) / 8;
    if (g.lda > (1 << 24) || (w4 ? *per > 32 : !g.w_vec)) return 0;
    const size_t sc = w4 ? (size_t)((*per * 16 * (128 / group) + 255) & ~255) * tiles * (zeros ? 2 : 1) : 0, sums = (size_t)32 * br * (16 * tiles + 4);
    const size_t held = g.a_vec ? 0 : (size_t)*per * br * 1024, stage = (size_t)((g.a_vec ? br : 0) + tiles * (w4 ? 1 : 2)) * 1024;
    auto bytes = [&](int n) { return 8 * (sc + (held + n * stage > sums ? held + n * stage : sums)); };
    const int64_t blocks = (((int64_t)g.N + tn - 1) / tn) * ((g.M + 8 * br - 1) / (8 * br));
    const size_t side = blocks <= 256 ? 1 : (blocks <= 512 ? 2 : 3);
    int n = *per < 4 ? *per : 4;
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
    g.a_vec = g.a_vec && g.K % 16 == 0;
    g.mp = ring_stages(g, W4, BR, NT, GATED, G, ZERO, &g.slab, &lds);
    if (g.mp == 0) return IBERT_ERR_NOT_IMPLEMENTED;
    g.chunks = (g.K + 127) / 128;
    return rows_pieces(kern, g, TM, 16 * NH, lds, stream, [] {
        static const KernelName name("rows_ring_kernel<%s, %d, %d, %d, %s, %s>", W4 ? "true" : "false", BR, NT, G, ZERO ? "true" : "false", GATED ? "true" : "false");
        return name.text;
    });
}

template <bool W4, int G, bool ZERO, bool GATED>
int launch_ring(const RowsArgs& g, const RowsPlan& plan, hipStream_t stream)
{
    constexpr int PER = GATED ? 2 : 1;
    if (plan.nt == 1) {
        if (plan.br == 1) return launch_ring_as<W4, 1, PER, G, ZERO, GATED>(g, stream);
        if (plan.br == 2) return launch_ring_as<W4, 2, PER, G, ZERO, GATED>(g, stream);
        if (plan.br == 4) return launch_ring_as<W4, 4, PER, G, ZERO, GATED>(g, stream);
        return launch_ring_as<W4, 8, PER, G, ZERO, GATED>(g, stream);
    }
    if constexpr (W4 && !GATED) if (plan.nt == 4) {
        if (plan.br == 1) return launch_ring_as<W4, 1, 4, G, ZERO, GATED>(g, stream);
        if (plan.br == 2) return launch_ring_as<W4, 2, 4, G, ZERO, GATED>(g, stream);
        return launch_ring_as<W4, 4, 4, G, ZERO, GATED>(g, stream);       // (8 rows' blocks: see launch_few_rows)
    }
    if (plan.br == 1) return launch_ring_as<W4, 1, 2 * PER, G, ZERO, GATED>(g, stream);
    if (plan.br == 2) return launch_ring_as<W4, 2, 2 * PER, G, ZERO, GATED>(g, stream);
    if (plan.br == 4) return launch_ring_as<W4, 4, 2 * PER, G, ZERO, GATED>(g, stream);
    return launch_ring_as<W4, 8, 2 * PER, G, ZERO, GATED>(g, stream);
}

template <bool W4, int G, int MT>
int launch_rows_of(const RowsArgs& g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream)
{
    if (gated) {
        if constexpr (!W4) return plan.nt == 2 ? launch_rows_as<W4, MT, 4, G, false, true>(g, plan, stream) : launch_rows_as<W4, MT, 2, G, false, true>(g, plan, stream);
        else if (plan.nt == 2) return zeros ? launch_rows_as<W4, MT, 4, G, true, true>(g, plan, stream) : launch_rows_as<W4, MT, 4, G, false, true>(g, plan, stream);
        else return zeros ? launch_rows_as<W4, MT, 2, G, true, true>(g, plan, stream) : launch_rows_as<W4, MT, 2, G, false, true>(g, plan, stream);
    }
    if constexpr (W4) {
        if (plan.nt == 2) return zeros ? launch_rows_as<W4, MT, 2, G, true, false>(g, plan, stream) : launch_rows_as<W4, MT, 2, G, false, false>(g, plan, stream);
        return zeros ? launch_rows_as<W4, MT, 1, G, true, false>(g, plan, stream) : launch_rows_as<W4, MT, 1, G, false, false>(g, plan, stream);
    }
    return IBERT_ERR_NOT_IMPLEMENTED;
}

#define IBERT_ROWS_UNIT(W4_, G_)                                                                                          \
    template <>                                                                                                           \
    int launch_rows<W4_, G_>(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream)                \
    {                                                                                                                     \
        if constexpr (W4_) {                                                                                              \
            if (plan.ring && gated) return zeros ? launch_ring<W4_, G_, true, true>(g, plan, stream) : launch_ring<W4_, G_, false, true>(g, plan, stream);      \
            if (plan.ring) return zeros ? launch_ring<W4_, G_, true, false>(g, plan, stream) : launch_ring<W4_, G_, false, false>(g, plan, stream);             \
        } else if (plan.ring) return launch_ring<W4_, G_, false, true>(g, plan, stream);                                  \
        if (plan.mt == 1) return launch_rows_of<W4_, G_, 1>(g, plan, zeros, gated, stream);                               \
        if (plan.mt == 2) return launch_rows_of<W4_, G_, 2>(g, plan, zeros, gated, stream);                               \
        return launch_rows_of<W4_, G_, 4>(g, plan, zeros, gated, stream);                                                 \
    }

}  // namespace ibert
