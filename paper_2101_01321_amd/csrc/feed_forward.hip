// The gated feed-forward block and the products with 4-bit weights: argument checks, the choice of the kernel, and the INT8 gated block's
// kernels for few rows.
#include "gated_stream.h"
#include "rows_launch.h"

namespace ibert {

template <> int launch_rows<true, 32>(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream);
template <> int launch_rows<true, 64>(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream);
template <> int launch_rows<true, 128>(RowsArgs g, const RowsPlan& plan, bool zeros, bool gated, hipStream_t stream);
IBERT_ROWS_UNIT(false, 128)

static int g_rows_tiles = -1, g_rows_rows = -1;

// Tiles of rows_ring_kernel: 8 br rows that hold M, up to 32 (of INT8 weights 64), by nt tiles of 16 channels (pairs of a gated block).  Wider tiles read A less
// often, and there must be enough of them.  us, tiles x blocks of rows, at N x K:
//   4 bits   1 row: 50000 x 1024 1x1 12.8 / 2x1 8.9, 12288 x 4096 8.1 / 9.0
//            64: 4096 x 12288 1x4 19.5 / 2x4 15.3, 4096 x 4096 8.0 / 8.3, 1024 x 4096 5.9 / 7.2
//            128: 4096 x 4096 2x4 10.3 / 4x4 11.4, 4096 x 12288 22.8 / 19.8;  256: 4096 x 4096 17.5 / 15.4, 50000 x 1024 79 / 83
//   pairs    64: 11008 x 4096 1x4 24.9 / 2x4 22.5, 4096 x 1024 6.1 / 6.6;  128: 4096 x 1024 9.3 / 8.5, 2730 x 1024 7.2 / 8.3
//   INT8     64: 8192 x 2048 1x4 14.4 / 2x8 13.0;  128: 11008 x 4096 48.2 / 42.1, 2730 x 1024 7.9 / 8.3;  256: 2730 x 1024 12.1 / 14.6
//   not there, by the rule / otherwise: 4 bits 2x8 64: 4096 x 12288 15.5 / 22.7, 256: 31.0 / 39.2, pairs 256: 11008 x 4096 56.5 / 67.9; 4 bits 4x1 8: 50000 x 1024 9.2 / 9.8,
//            4x2 16: 11.0 / 13.0; pairs 2x1 8: 11008 x 4096 11.7 / 13.5, 2x2 16: 13.1 / 14.7, INT8 pairs 2x2 16: 19.7 / 21.7, 2x4 32: 22.7 / 26.1, 1x8 64: 2730 x 1024 5.3 / 5.6
static void plan_ring(RowsPlan& p, int32_t M, int32_t N, int32_t K, bool w4, bool gated)
{
    auto blocks = [&](int nt, int br) { return ((int64_t)N + 16 * nt - 1) / (16 * nt) * (((int64_t)M + 8 * br - 1) / (8 * br)); };
    p.br = M <= 8 ? 1 : (M <= 16 ? 2 : 4);
    p.nt = 1;
    if (!w4) {
        const int64_t b = blocks(2, 8);
        if (M > 32 && 4 * b >= 3 * 256 * ((b + 255) / 256)) {
            p.nt = 2;
            p.br = 8;
        }
    } else if (gated) {
        if (p.br == 4 && blocks(1, 4) >= 1024) p.nt = 2;
    } else if (p.br == 4) {
        if (K >= 2048 && blocks(4, 4) >= (K >= 8192 ? 256 : 512)) p.nt = 4;
        else if (blocks(1, 4) >= 512) p.nt = 2;
    } else if (blocks(1, p.br) > 1536) p.nt = 2;
}

// The kernel of an INT8 gated block: 0 rows_ring_kernel, else the persistent one's tile; by what rounds of its workgroups over the chip's 256 units are expected to take, us, from
// K / 1024 = k: a round of 64 x 32 rings 4 + 2.8 k behind the first 1.2, of 128 x 128 tiles 5.5 + 6.3 k, of 256 x 128 tiles 9.3 + 8.4 k, of 128 x 64 tiles 5.0 + 5.6 k where there
// is one to a unit and 5.5 + 7 k where there are two.
// Measured, us, rings / narrow / low / tall: 128 x 768 x 2048 4.8 / 8.8 / 10.9 / 15.7, 128 x 1024 x 4096 8.1 / 9.6 / 12.0 / 17.7, 64 x 4096 x 11008 31.3 / 27.2 / 34.5 / 43.0,
// 256 x 1024 x 4096 14.9 / 9.3 / 11.9 / 17.8, 128 x 2048 x 8192 20.2 / 15.8 / 20.0 / 26.5, 1000 x 768 x 2048 - / 9.6 / 11.5 / 16.1, 512 x 1024 x 4096 - / 11.2 / 13.1 / 18.2,
// 1024 x 4096 x 4096 - / 39.5 / 36.4 / 45.8, 2741 x 1024 x 4096 - / 33.8 / 34.0 / 36.3, 2048 x 4096 x 11008 - / 207 / 220 / 166, 8192 x 4096 x 12288 - / 882 / 787 / 652.
static int plan_gated(int32_t M, int32_t F, int32_t K)
{
    auto tiles = [&](int rows, int channels) { return (((int64_t)M + rows - 1) / rows) * (((int64_t)F + channels - 1) / channels); };
    auto ns = [&](int64_t fixed, int64_t per_k, int64_t n) { return (n + 255) / 256 * (fixed + per_k * K / 1024); };
    const int64_t ring = 1200 + ns(4000, 2800, tiles(64, 32)), low = ns(5500, 6300, tiles(128, 128)), tall = ns(9300, 8400, tiles(256, 128));
    const int64_t n = tiles(128, 64), odd = n % 512 > 0 && n % 512 <= 256, narrow = (odd ? ns(5000, 5600, 1) : 0) + ns(5500, 7000, ((n + 511) / 512 - odd) * 256);
    if (M <= 32 || (ring <= narrow && ring <= low && ring <= tall)) return 0;
    if (narrow < low && narrow < tall) return GATED_NARROW;
    return low <= tall ? GATED_LOW : GATED_TALL;
}

static int launch_few_rows(RowsArgs& g, bool w4, int32_t group, bool zeros, bool gated, hipStream_t stream)
{
    g.chunks = (g.K + 127) / 128;
    g.per = (g.chunks + 7) / 8;
    RowsPlan p{};
    plan_ring(p, g.M, g.N, g.K, w4, gated);
    if (g_rows_tiles > 0) {
        // (of the tiles that there are: see launch_ring)
        if (g_rows_rows > 0) p.br = w4 && g_rows_rows > 4 ? 4 : g_rows_rows;
        if (!w4) p.nt = p.br == 8 ? 2 : 1;
        else if (gated) p.nt = g_rows_tiles > 1 && p.br == 4 ? 2 : 1;
        else p.nt = g_rows_tiles == 4 && p.br < 4 ? 2 : g_rows_tiles;
    }
    size_t lds;
    auto fits = [&] { return ring_stages(g, w4, p.br, (gated ? 2 : 1) * p.nt, gated, group, zeros, &lds) > 0; };
    const int32_t rows = p.br, tiles = p.nt;
    while (p.nt > 1 && !fits()) p.nt >>= 1;
    while (p.br > 1 && !fits()) p.br >>= 1;
    p.ring = g_rows_rows != 0 && fits();
    if (!p.ring) {
        p.br = rows;
        p.nt = tiles;
    }
    if (!w4) return launch_rows<false, 128>(g, p, false, true, stream);
    if (group == 32) return launch_rows<true, 32>(g, p, zeros, gated, stream);
    if (group == 64) return launch_rows<true, 64>(g, p, zeros, gated, stream);
    return launch_rows<true, 128>(g, p, zeros, gated, stream);
}

// (128 bits: whatever leading dimensions and rows are given, no sum here passes them)
typedef unsigned __int128 extent;
static bool overlap(const void* a, extent abytes, const void* b, extent bbytes)
{
    const extent x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + bbytes && y < x + abytes;
}
// bytes from the first to the last element of `rows` >= 1 rows of n elements
static extent span(int64_t rows, int64_t ld, int64_t n, int64_t elem) { return ((extent)(rows - 1) * (extent)ld + (extent)n) * (extent)elem; }

static int check_gate(const ibert_gate_params& p)
{
    if (p.activation != IBERT_GATE_SILU && p.activation != IBERT_GATE_GELU) return IBERT_ERR_PARAM_RANGE;
    if (p.activation == IBERT_GATE_GELU) {
        const int rc = check_gelu(p.gelu);
        if (rc) return rc;
    }
    return dyadic_ok(p.out_dy) ? IBERT_OK : IBERT_ERR_PARAM_RANGE;
}

// Sizes and constants of a gated block; *empty: there is nothing to do.
static int check_gated(const ibert_gated_desc* d, const int8_t* A, const int32_t* mult, const int32_t* shift, const int8_t* C, bool* empty)
{
    *empty = false;
    if (!d) return IBERT_ERR_NULL;
    if (d->M < 0 || d->F < 0 || d->K < 1 || d->K > (1 << 17) || d->F > (1 << 24)) return IBERT_ERR_SHAPE;
    const int rc = check_gate(d->gate);
    if (rc) return rc;
    if (d->lda < d->K || d->ldc < d->F) return IBERT_ERR_SHAPE;
    *empty = d->M == 0 || d->F == 0;
    if (*empty) return IBERT_OK;
    if (!A || !mult || !shift || !C) return IBERT_ERR_NULL;
    if (overlap(C, span(d->M, d->ldc, d->F, 1), A, span(d->M, d->lda, d->K, 1))) return IBERT_ERR_SHAPE;
    return IBERT_OK;
}

static int check_w4(const ibert_w4_weights* w)
{
    if (!w) return IBERT_ERR_NULL;
    if (w->group != 32 && w->group != 64 && w->group != 128) return IBERT_ERR_PARAM_RANGE;
    if (!w->w || !w->scales) return IBERT_ERR_NULL;
    if (!aligned(w->w, 16) || !aligned(w->scales, 4) || (w->zeros && !aligned(w->zeros, 4))) return IBERT_ERR_ALIGN;
    return IBERT_OK;
}

static RowsArgs rows_args(const int8_t* A, int64_t lda, int32_t M, int32_t N, int32_t K, const int32_t* bias, const int32_t* mult, const int32_t* shift,
                          void* C, int64_t ldc)
{
    RowsArgs g{};
    g.A = A; g.lda = lda; g.M = M; g.N = N; g.K = K;
    g.bias = bias; g.mult = mult; g.shift = shift;
    g.C = C; g.ldc = ldc;
    g.a_vec = aligned(A, 16) && lda % 16 == 0 && K % 16 == 0;
    return g;
}

}  // namespace ibert

extern "C" void ibert_rows_override(int32_t tiles, int32_t rows)
{
    ibert::g_rows_tiles = tiles;
    ibert::g_rows_rows = rows;
}

extern "C" int ibert_gemm_i8_gated(const ibert_gated_desc* desc, const int8_t* A, const int8_t* W, const int32_t* bias,
                                   const int32_t* mult, const int32_t* shift, int8_t* C, void* stream)
{
    bool empty;
    const int rc = ibert::check_gated(desc, A, mult, shift, C, &empty);
    if (rc) return rc;
    if (desc->ldw < desc->K) return IBERT_ERR_SHAPE;
    if (empty) return IBERT_OK;
    if (!W) return IBERT_ERR_NULL;
    const ibert_gated_desc& d = *desc;
    if (ibert::overlap(C, ibert::span(d.M, d.ldc, d.F, 1), W, ibert::span(2 * (int64_t)d.F, d.ldw, d.K, 1))) return IBERT_ERR_SHAPE;
    int tile = 0;
    if (ibert::g_rows_tiles < 0) tile = ibert::plan_gated(d.M, d.F, d.K);
    else if (ibert::g_rows_tiles == 0) tile = ibert::g_rows_rows == 1 ? ibert::GATED_LOW : (ibert::g_rows_rows == 3 ? ibert::GATED_NARROW : ibert::GATED_TALL);
    if (tile > 0 && ibert::gated_stream_ok(d, A, W))
        return ibert::launch_gated_stream(d, A, W, bias, mult, shift, C, tile, static_cast<hipStream_t>(stream));
    ibert::RowsArgs g = ibert::rows_args(A, d.lda, d.M, d.F, d.K, bias, mult, shift, C, d.ldc);
    g.w[0] = W;
    g.ldw = d.ldw;
    g.w_vec = ibert::aligned(W, 16) && d.ldw % 16 == 0 && d.K % 16 == 0 && d.ldw <= (1 << 26);
    g.gate = ibert::gate_const(d.gate);
    return ibert::launch_few_rows(g, false, 128, false, true, static_cast<hipStream_t>(stream));
}

extern "C" int ibert_gemm_w4_gated(const ibert_gated_desc* desc, const int8_t* A, const ibert_w4_weights* gate, const ibert_w4_weights* up,
                                   const int32_t* bias, const int32_t* mult, const int32_t* shift, int8_t* C, void* stream)
{
    bool empty;
    int rc = ibert::check_gated(desc, A, mult, shift, C, &empty);
    if (rc) return rc;
    if (empty) return IBERT_OK;
    rc = ibert::check_w4(gate);
    if (rc) return rc;
    rc = ibert::check_w4(up);
    if (rc) return rc;
    if (gate->group != up->group || (gate->zeros != nullptr) != (up->zeros != nullptr)) return IBERT_ERR_PARAM_RANGE;
    const ibert_gated_desc& d = *desc;
    const ibert::extent wbytes = ibert_w4_bytes(d.F, d.K), cbytes = ibert::span(d.M, d.ldc, d.F, 1);
    if (ibert::overlap(C, cbytes, gate->w, wbytes) || ibert::overlap(C, cbytes, up->w, wbytes)) return IBERT_ERR_SHAPE;
    ibert::RowsArgs g = ibert::rows_args(A, d.lda, d.M, d.F, d.K, bias, mult, shift, C, d.ldc);
    g.w[0] = gate->w; g.w[1] = up->w;
    g.scales[0] = gate->scales; g.scales[1] = up->scales;
    g.zeros[0] = gate->zeros; g.zeros[1] = up->zeros;
    g.gate = ibert::gate_const(d.gate);
    return ibert::launch_few_rows(g, true, gate->group, gate->zeros != nullptr, true, static_cast<hipStream_t>(stream));
}

extern "C" int ibert_gemm_w4_requant(const ibert_w4_desc* desc, const int8_t* A, const ibert_w4_weights* weights, const int32_t* bias,
                                     const int32_t* mult, const int32_t* shift, const int8_t* residual, void* C, void* stream)
{
    if (!desc) return IBERT_ERR_NULL;
    const ibert_w4_desc& d = *desc;
    if (d.M < 0 || d.N < 0 || d.K < 1 || d.K > (1 << 17) || d.N > (1 << 24)) return IBERT_ERR_SHAPE;
    if (d.out_dtype != IBERT_I8 && d.out_dtype != IBERT_I32 && d.out_dtype != IBERT_I16) return IBERT_ERR_PARAM_RANGE;
    if (d.out_clamp < 0 || (d.out_dtype == IBERT_I8 && d.out_clamp > 127) || (d.out_dtype == IBERT_I16 && d.out_clamp > 32767)) return IBERT_ERR_PARAM_RANGE;
    if (residual && !ibert::dyadic_ok(d.residual_dy)) return IBERT_ERR_PARAM_RANGE;
    if (d.lda < d.K || d.ldc < d.N || (residual && d.ldr < d.N)) return IBERT_ERR_SHAPE;
    if (d.M == 0 || d.N == 0) return IBERT_OK;
    if (!A || !mult || !shift || !C) return IBERT_ERR_NULL;
    const int rc = ibert::check_w4(weights);
    if (rc) return rc;
    const int64_t elem = d.out_dtype == IBERT_I8 ? 1 : (d.out_dtype == IBERT_I16 ? 2 : 4);
    const ibert::extent cbytes = ibert::span(d.M, d.ldc, d.N, elem);
    if (ibert::overlap(C, cbytes, A, ibert::span(d.M, d.lda, d.K, 1)) || ibert::overlap(C, cbytes, weights->w, ibert_w4_bytes(d.N, d.K)) ||
        (residual && ibert::overlap(C, cbytes, residual, ibert::span(d.M, d.ldr, d.N, 1)))) return IBERT_ERR_SHAPE;
    ibert::RowsArgs g = ibert::rows_args(A, d.lda, d.M, d.N, d.K, bias, mult, shift, C, d.ldc);
    g.w[0] = weights->w;
    g.scales[0] = weights->scales;
    g.zeros[0] = weights->zeros;
    g.R = residual; g.ldr = d.ldr;
    g.res_m = d.residual_dy.m; g.res_s = d.residual_dy.s;
    g.out_dtype = d.out_dtype; g.out_clamp = d.out_clamp;
    return ibert::launch_few_rows(g, true, weights->group, weights->zeros != nullptr, false, static_cast<hipStream_t>(stream));
}
