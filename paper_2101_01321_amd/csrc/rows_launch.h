// How a product of few rows is laid out (RowsPlan), and its launch.  One unit per group size instantiates launch_rows.
#pragma once
#include "rows_kernel.h"

namespace ibert {

// rows of a workgroup / 16 (1, 2, 4); tiles of 16 channels to a wavefront, of each matrix of a gated block (1, 2); log2 of its groups of channels
struct RowsPlan {
    int32_t mt, nt, cg;
};

template <bool W4, int G>
int launch_rows(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream);

constexpr int ROWS_LDS = 163840;

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
    const int64_t M = g.M;
    const int32_t rows = M < 16 * MT ? (int32_t)M : 16 * MT;
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
    const int64_t across = (g.N + (16 * NH << g.cg) - 1) / (16 * NH << g.cg);
    // (a launch may have 2^32 threads at most: pieces of rows)
    const int64_t down = (M + 16 * MT - 1) / (16 * MT), most_down = (1 << 22) / across < 1 ? 1 : (1 << 22) / across;
    const int8_t *A = g.A, *R = g.R;
    char* C = static_cast<char*>(g.C);
    const int64_t elem = g.out_dtype == IBERT_I8 ? 1 : (g.out_dtype == IBERT_I16 ? 2 : 4);
    for (int64_t d0 = 0; d0 < down; d0 += most_down) {
        const int64_t m0 = d0 * 16 * MT, n = down - d0 < most_down ? down - d0 : most_down;
        g.A = A + m0 * g.lda;
        g.R = R ? R + m0 * g.ldr : nullptr;
        g.C = C + m0 * g.ldc * elem;
        g.M = (int32_t)(M - m0 < n * 16 * MT ? M - m0 : n * 16 * MT);
        g.down = (int32_t)n;
        g.across = (int32_t)across;
        const int64_t blocks = (across + 7) / 8 * 8 * n;
        hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(ROWS_THREADS), lds, stream, g);
        IBERT_LAUNCH_CHECK("rows_kernel");
    }
    static const KernelName name("rows_kernel<%s, %d, %d, %d, %s, %s>", W4 ? "true" : "false", MT, NT, G, ZERO ? "true" : "false", GATED ? "true" : "false");
    g_last_kernel = name.text;
    return IBERT_OK;
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
        if (plan.mt == 1) return launch_rows_of<W4_, G_, 1>(g, plan, zeros, gated, stream);                               \
        if (plan.mt == 2) return launch_rows_of<W4_, G_, 2>(g, plan, zeros, gated, stream);                               \
        return launch_rows_of<W4_, G_, 4>(g, plan, zeros, gated, stream);                                                 \
    }

}  // namespace ibert
