// Causal attention of query rows over an INT8 key/value cache in pages (ibert_paged_attention_i).
//
// Rows: the query heads of a sequence that share a key head are rows of one problem, n queries x (heads_q / heads_kv) heads,
// the query outermost; 16 of them are a tile.  Scores: v_mfma_i32_16x16x64_i8 with 16 keys as the first operand and the tile's
// rows as the second; lane l then holds, for row l % 16, the keys 16 i + 4 (l / 16) + r of 64.  Their weights, 15 bits in
// two INT8 halves (w = 256 h + l), packed four to a dword i, are the second operand of the product with the values as they
// stand: the cache keeps 64 tokens of a channel in exactly that order, so that neither scores nor weights cross lanes.
// The weights are relative to the row's maximum and cannot be rescaled exactly, so the maximum is made first, over the raw
// accumulators (the distance is monotone in them), and the scores are made a second time.
#include "common.h"
#include "ibert_testing.h"

namespace ibert {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int PA_MOST_KEYS = 131072;

struct PagedArgs {
    const int8_t *q, *k, *v;
    int8_t* out;
    const int32_t *table, *q_start, *kv_len;
    int64_t ld_q, ld_out;
    int32_t heads_q, heads_kv, group, log_page, num_pages, max_pages, rows, max_q, keys;   // keys: most that a sequence can have
    int32_t window, sinks;
    int32_t only;              // 1: the sequences of one row, 2: the others, 0: all
    int32_t packed;            // sequences, where the prompt kernel's workgroups find theirs by counting; else 0
    uint32_t group_magic, s_m;
    int32_t s_l, s_r;          // DY(d) = (((uint64)(d << s_l) * s_m + s_rnd) >> 32) >> s_r
    uint64_t s_rnd;
    int32_t s_s;               // the shift of DY; less 32 where that is not negative
    ibert_dyadic out_dy;
};

// Query of the flat row n.
__device__ __forceinline__ int32_t group_of(const PagedArgs& a, int32_t n) { return udiv_fix(n, a.group, a.group_magic); }

// Is a sequence of n rows one that this launch leaves to another?
__device__ __forceinline__ bool left_out(const PagedArgs& a, int32_t n) { return a.only && (a.only == 1) != (n == 1); }

// What one workgroup works on: 16 rows of one sequence and key head.
struct Tile {
    int32_t row0, n;           // first query row of the sequence in q; its queries
    int32_t pos0;              // position of its first query
    int32_t kv;                // keys
    int32_t first, count;      // the tile's first flat row; how many rows it has
    int32_t low, high;         // positions of its first and last query
    int32_t sink_blocks, from, blocks;   // 64-key blocks to look at: [0, sink_blocks) and from [from ..), blocks in all
};

__device__ __forceinline__ Tile tile_of(const PagedArgs& a, int b, int tile, int tile_rows)
{
    Tile t;
    int32_t r0 = b, r1 = b + 1;
    if (a.q_start) {
        r0 = clamp_i32(a.q_start[b], 0, a.rows);
        r1 = clamp_i32(a.q_start[b + 1], r0, a.rows);
    }
    t.row0 = r0; t.n = r1 - r0;
    t.kv = clamp_i32(a.kv_len[b], 0, a.keys);
    t.pos0 = t.kv - t.n;
    t.first = tile * tile_rows;
    const int64_t left = (int64_t)(t.n < a.max_q ? t.n : a.max_q) * a.group - t.first;
    t.count = left < tile_rows ? (int32_t)(left < 0 ? 0 : left) : tile_rows;
    if (left_out(a, t.n)) t.count = 0;
    t.low = t.pos0 + group_of(a, t.first);
    t.high = t.pos0 + group_of(a, t.first + (t.count > 0 ? t.count - 1 : 0));
    const int32_t end = t.high < 0 ? 0 : (t.high >> 6) + 1;
    int32_t from = 0, sb = 0;
    if (a.window > 0 && t.low >= a.window) {
        from = (t.low - a.window + 1) >> 6;
        sb = (a.sinks >> 6) + ((a.sinks & 63) != 0);
        if (sb >= from) { sb = 0; from = 0; }
    }
    t.sink_blocks = sb; t.from = from; t.blocks = sb + (end > from ? end - from : 0);
    return t;
}

__device__ __forceinline__ int block_at(const Tile& t, int x) { return x < t.sink_blocks ? x : x - t.sink_blocks + t.from; }

// Offset of a block of 64 tokens in k and in v.
template <int D>
__device__ __forceinline__ int64_t block_offset(const PagedArgs& a, int b, int h, int block)
{
    const int lp = a.log_page - 6;
    // (a scalar load: no wait for it counts the requests of keys and values that are on their way)
    const auto* entries = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)a.table;
    int32_t page = entries[(int64_t)b * a.max_pages + (block >> lp)];
    page = clamp_i32(page, 0, a.num_pages - 1);
    return ((((int64_t)page * a.heads_kv + h) << lp) + (block & ((1 << lp) - 1))) * (64 * D);
}

// May every row of the tile see every key of the block?
__device__ __forceinline__ bool whole_block(const PagedArgs& a, const Tile& t, int block)
{
    // (no branches: the tests stand beside matrix instructions, which a branch would part from what is to run beside them)
    return (64 * block + 63 <= t.low) & ((a.window == 0) | (64 * block > t.high - a.window) | (64 * block + 63 < a.sinks));
}
__device__ __forceinline__ bool visible(const PagedArgs& a, int key, int pos)
{
    return key <= pos && (a.window == 0 || key > pos - a.window || key < a.sinks);
}

// Weight of a key whose raw score is d under the row's largest.
__device__ __forceinline__ uint32_t weight_of(const PagedArgs& a, uint32_t d)
{
    uint32_t e = (uint32_t)(((uint64_t)(d << a.s_l) * a.s_m + a.s_rnd) >> 32) >> a.s_r;
    e = e < 1024u ? e : 1024u;
    const uint32_t z = e >> 6, f = 124u - (e & 63u);
    return (umad24(f, f, 8180u) + ((1u << z) >> 1)) >> z;
}

// Operands of a block of 64 keys: K as four tiles of 16 keys, V as D / 16 tiles of 16 channels.
template <int D>
__device__ __forceinline__ void load_k(const PagedArgs& a, int64_t at, int lane, v4i (&kf)[D / 16])
{
#pragma unroll
    for (int i = 0; i < D / 16; ++i) kf[i] = *reinterpret_cast<const v4i*>(a.k + at + i * 1024 + lane * 16);
}
template <int D>
__device__ __forceinline__ void load_v(const PagedArgs& a, int64_t at, int lane, v4i (&vf)[D / 16])
{
#pragma unroll
    for (int i = 0; i < D / 16; ++i) vf[i] = *reinterpret_cast<const v4i*>(a.v + at + i * 1024 + lane * 16);
}

// Raw scores of the lane's row; keys that it may not see: INT32_MIN.
template <int D>
__device__ __forceinline__ void block_scores(const PagedArgs& a, const Tile& t, int block, int pos, int g, const v4i (&kf)[D / 16], const v4i (&qf)[D / 64], v4i (&s)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = v4i{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < D / 64; ++j) s[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[i * (D / 64) + j], qf[j], s[i], 0, 0, 0);
    }
    if (!whole_block(a, t, block)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!visible(a, 64 * block + 16 * i + 4 * g + r, pos)) s[i][r] = INT32_MIN;
    }
}

__device__ __forceinline__ int32_t largest(const v4i (&s)[4], int32_t mx)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = mx > s[i][r] ? mx : s[i][r];
    return mx;
}

// Weights of a block as MFMA operands, in two halves; sum: of the weights.
__device__ __forceinline__ void block_weights(const PagedArgs& a, const v4i (&s)[4], int32_t mx, v4i& wh, v4i& wl, uint32_t& sum)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            w[r] = weight_of(a, (uint32_t)mx - (uint32_t)s[i][r]);
            w[r] = s[i][r] == INT32_MIN ? 0 : w[r];
            sum += w[r];
        }
        wl[i] = (int32_t)pack4_perm((int32_t)w[0], (int32_t)w[1], (int32_t)w[2], (int32_t)w[3]);
        wh[i] = (int32_t)pack4_perm((int32_t)((w[0] + 128) >> 8), (int32_t)((w[1] + 128) >> 8), (int32_t)((w[2] + 128) >> 8), (int32_t)((w[3] + 128) >> 8));
    }
}

// floor(2^48 / W), and 0 for a row that sees nothing.
__device__ __forceinline__ uint64_t reciprocal(uint32_t W) { return W ? ((uint64_t)1 << 48) / W : 0; }
__device__ __forceinline__ int8_t finished(const PagedArgs& a, int64_t N, uint64_t R)
{
    return (int8_t)clamp_i64_to_i32(dyadic64((int32_t)((N * (int64_t)R) >> 32), a.out_dy.m, a.out_dy.s), 127);
}

// The row of a tile that a lane's column stands for (columns behind the last row repeat it), and its queries as operand.
template <int D>
__device__ __forceinline__ void tile_row(const PagedArgs& a, const Tile& t, int h, int c, int g, int& pos, v4i (&qf)[D / 64])
{
    const int flat = t.first + (c < t.count ? c : t.count - 1), qi = group_of(a, flat);
    const int8_t* src = a.q + (int64_t)(t.row0 + qi) * a.ld_q + (h * a.group + (flat - qi * a.group)) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) qf[j] = *reinterpret_cast<const v4i*>(src + 64 * j);
    pos = t.pos0 + qi;
}

// ---- any number of rows, no workspace: the scores are made twice -----------------------------------------------------
// NW wavefronts take every NW-th block of keys.  Eight, which ask for a block ahead (177 registers at width 128: one workgroup on a unit), where each workgroup has a
// unit to itself; else four, which leave it to the other workgroups on the unit.  us, four / eight, 8 key heads of width 128 on 4000 keys: 32 workgroups 25.9 / 21.9, 128
// 33.1 / 25.1, 256 44.1 / 38.9, 384 68.7 / 72.0, 512 73.9 / 90.7; 16 heads of width 64, 192 31.2 / 26.5.  Bound: latency up to there, then HBM or L2.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 2 : 3) void paged_attention_kernel(PagedArgs a)
{
    constexpr int NJ = D / 64, ND = D / 16;
    constexpr bool AHEAD = NW == 8;
    __shared__ int32_t s_max[NW][16];
    __shared__ int32_t s_hi[D * 16], s_lo[D * 16], s_w[32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int h = blockIdx.x, b = blockIdx.y;
    const Tile t = tile_of(a, b, blockIdx.z, 16);
    if (t.count == 0) return;
    for (int i = tid; i < D * 16; i += 64 * NW) { s_hi[i] = 0; s_lo[i] = 0; }
    if (tid < 32) s_w[tid] = 0;
    int pos;
    v4i qf[NJ];
    tile_row<D>(a, t, h, c, g, pos, qf);
    const int n = t.blocks;
    auto offset = [&](int x) { return block_offset<D>(a, b, h, block_at(t, x)); };
    const auto larger = [](int32_t p, int32_t q) { return p > q ? p : q; };

    v4i f0[ND], f1[ND];
    int32_t mx = INT32_MIN;
    auto compare = [&](int x, const v4i (&k)[ND]) {
        v4i s[4];
        block_scores<D>(a, t, block_at(t, x), pos, g, k, qf, s);
        mx = largest(s, mx);
    };
    if constexpr (AHEAD) {
        int x = wave;
        if (x < n) load_k<D>(a, offset(x), lane, f0);
        while (x < n) {
            if (x + NW < n) load_k<D>(a, offset(x + NW), lane, f1);
            compare(x, f0);
            x += NW;
            if (x >= n) break;
            if (x + NW < n) load_k<D>(a, offset(x + NW), lane, f0);
            compare(x, f1);
            x += NW;
        }
        if (wave < n) load_k<D>(a, offset(wave), lane, f0);
    } else {
        for (int x = wave; x < n; x += NW) {
            load_k<D>(a, offset(x), lane, f0);
            compare(x, f0);
        }
    }
    mx = combine_rows32(combine_rows16(mx, larger), larger);
    if (g == 0) s_max[wave][c] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) mx = larger(mx, s_max[w][c]);

    v4i hi[ND], lo[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) { hi[i] = v4i{0, 0, 0, 0}; lo[i] = v4i{0, 0, 0, 0}; }
    uint32_t sum = 0;
    for (int x = wave; x < n; x += NW) {
        v4i s[4], wh, wl;
        if (!AHEAD) load_k<D>(a, offset(x), lane, f0);
        load_v<D>(a, offset(x), lane, f1);
        block_scores<D>(a, t, block_at(t, x), pos, g, f0, qf, s);
        if (AHEAD && x + NW < n) load_k<D>(a, offset(x + NW), lane, f0);
        block_weights(a, s, mx, wh, wl, sum);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            hi[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f1[i], wh, hi[i], 0, 0, 0);
            lo[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f1[i], wl, lo[i], 0, 0, 0);
        }
    }
    // whole numbers: the order of these additions changes nothing
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            atomicAdd(&s_hi[(16 * i + 4 * g + r) * 16 + c], hi[i][r]);
            atomicAdd(&s_lo[(16 * i + 4 * g + r) * 16 + c], lo[i][r]);
        }
    atomicAdd(&s_w[c], (int32_t)sum);
    __syncthreads();
    if (tid < 16) {
        const uint64_t R = reciprocal((uint32_t)s_w[tid]);
        s_w[tid] = (int32_t)(uint32_t)R;
        s_w[16 + tid] = (int32_t)(uint32_t)(R >> 32);
    }
    __syncthreads();
    for (int e = tid; e < D * 16; e += 64 * NW) {
        const int r = e / D, d = e - r * D;
        if (r >= t.count) break;
        const int f = t.first + r, qr = group_of(a, f), hd = h * a.group + (f - qr * a.group);
        const int64_t N = (int64_t)s_hi[d * 16 + r] * 256 + s_lo[d * 16 + r];
        a.out[(int64_t)(t.row0 + qr) * a.ld_out + hd * D + d] = finished(a, N, ((uint64_t)(uint32_t)s_w[16 + r] << 32) | (uint32_t)s_w[r]);
    }
}

// ---- few rows, one launch: a workgroup for each sequence, key head and tile, scores in LDS --------------------------------
// K once, the scores into LDS, the maximum over the workgroup, then V once.  LDS: scores [held][64 blocks], then the sums [held][D], high
// and low halves.  Bound: HBM.  64 sequences of up to 4096 keys, 8 key heads of width 128 with 4 queries each: 342 MB in 67.7 us (5.05 TB/s; a copy reaches 5.17);
// 32 x 1025 visible keys in 16 heads of width 64: 67 MB in 16.4 us (4.1 TB/s); few keys: the launch and four dependent trips to memory, 5.2 us for 77.
constexpr int PW_NW = 8;
template <int D>
__global__ __launch_bounds__(64 * PW_NW, 2) void paged_row_kernel(PagedArgs a, int32_t held, int32_t room)
{
    constexpr int ND = D / 16, NW = PW_NW;
    extern __shared__ __attribute__((aligned(16))) int32_t pw_lds[];
    __shared__ int32_t s_max[NW][16];
    __shared__ uint32_t s_w[16];
    __shared__ uint64_t s_r[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int h = blockIdx.x, b = blockIdx.y;
    const Tile t = tile_of(a, b, blockIdx.z, 16);
    if (t.count == 0) return;
    int32_t* const s_hi = pw_lds + held * 64 * room;
    int32_t* const s_lo = s_hi + held * D;
    int pos;
    v4i qf[D / 64];
    tile_row<D>(a, t, h, c, g, pos, qf);
    const int n = t.blocks < room ? t.blocks : room;       // (room is made for all there can be)
    auto offset = [&](int x) { return block_offset<D>(a, b, h, block_at(t, x)); };
    const int mine = (c < held ? c : held - 1) * 64 * room + g * 16;
    const auto larger = [](int32_t p, int32_t q) { return p > q ? p : q; };

    v4i f0[ND], f1[ND];
    int32_t mx = INT32_MIN;
    auto score = [&](int x, const v4i (&k)[ND]) {
        v4i s[4];
        block_scores<D>(a, t, block_at(t, x), pos, g, k, qf, s);
        mx = largest(s, mx);
        if (c < held) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<v4i*>(pw_lds + mine + x * 64 + 4 * i) = s[i];
        }
    };
    int x = wave;
    if (x < n) load_k<D>(a, offset(x), lane, f0);
    while (x < n) {
        if (x + NW < n) load_k<D>(a, offset(x + NW), lane, f1);
        score(x, f0);
        x += NW;
        if (x >= n) break;
        if (x + NW < n) load_k<D>(a, offset(x + NW), lane, f0);
        score(x, f1);
        x += NW;
    }
    x = wave;
    if (x < n) load_v<D>(a, offset(x), lane, f0);
    mx = combine_rows32(combine_rows16(mx, larger), larger);
    if (g == 0) s_max[wave][c] = mx;
    for (int i = tid; i < 2 * held * D; i += 64 * NW) s_hi[i] = 0;
    if (tid < 16) s_w[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) mx = larger(mx, s_max[w][c]);

    v4i hi[ND], lo[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) { hi[i] = v4i{0, 0, 0, 0}; lo[i] = v4i{0, 0, 0, 0}; }
    uint32_t sum = 0;
    auto value = [&](int x, const v4i (&v)[ND]) {
        v4i s[4], wh, wl;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = *reinterpret_cast<const v4i*>(pw_lds + mine + x * 64 + 4 * i);
        block_weights(a, s, mx, wh, wl, sum);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            hi[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i], wh, hi[i], 0, 0, 0);
            lo[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i], wl, lo[i], 0, 0, 0);
        }
    };
    while (x < n) {
        if (x + NW < n) load_v<D>(a, offset(x + NW), lane, f1);
        value(x, f0);
        x += NW;
        if (x >= n) break;
        if (x + NW < n) load_v<D>(a, offset(x + NW), lane, f0);
        value(x, f1);
        x += NW;
    }
    // whole numbers: the order of these additions changes nothing
    if (c < held) {
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                atomicAdd(&s_hi[c * D + 16 * i + 4 * g + r], hi[i][r]);
                atomicAdd(&s_lo[c * D + 16 * i + 4 * g + r], lo[i][r]);
            }
        atomicAdd(&s_w[c], sum);
    }
    __syncthreads();
    if (tid < held) s_r[tid] = reciprocal(s_w[tid]);
    __syncthreads();
    for (int e = tid; e < t.count * D; e += 64 * NW) {
        const int r = e / D, d = e - r * D, f = t.first + r, qr = group_of(a, f), hd = h * a.group + (f - qr * a.group);
        a.out[(int64_t)(t.row0 + qr) * a.ld_out + hd * D + d] = finished(a, (int64_t)s_hi[e] * 256 + s_lo[e], s_r[r]);
    }
}

// ---- few rows on many keys: three launches, the keys of a tile of rows split into chunks ---------------------------------
// Scores and each chunk's maximum; weights, sums over the chunk, with the maximum of all chunks; the chunks' sums joined.  (The weights need the whole row's
// maximum, so there is a launch between the scores and them.)  Bound: HBM.  One sequence of 131071 keys, 8 key heads of width 128 with 4 queries each: 30.1, 32.4 and
// 4.6 us, K's and V's 134 MB each at 4.5 and 4.1 TB/s with 17 MB of scores between them.
struct SplitArgs {
    PagedArgs p;
    int32_t tiles, splits, chunk;      // row tiles of a key head; chunks of at most `chunk` blocks
    int32_t blocks, held;              // room in `scores`: blocks, and rows of a tile (min(16, rows there are))
    int32_t* maxima;                   // [batch][key head][tile][split][16]
    uint32_t* sums;                    // the same
    int64_t* parts;                    // [..][split][held][D]
    int32_t* scores;                   // [..][blocks][held][64], of a row the four lanes' 16 values one after the other
};

struct SplitAt {
    int b, h, split, x0, x1;
    int64_t index;                     // of (sequence, key head, tile)
    Tile t;
};
__device__ __forceinline__ SplitAt split_at(const SplitArgs& a, int split, int ht, int b)
{
    SplitAt s;
    s.b = b; s.split = split;
    s.h = ht / a.tiles;
    s.index = (int64_t)b * a.p.heads_kv * a.tiles + ht;
    s.t = tile_of(a.p, b, ht - s.h * a.tiles, 16);
    s.x0 = split * a.chunk;
    s.x1 = s.x0 + a.chunk < s.t.blocks ? s.x0 + a.chunk : s.t.blocks;
    return s;
}
__device__ __forceinline__ int splits_used(const SplitArgs& a, const Tile& t) { return (t.blocks + a.chunk - 1) / a.chunk; }

template <int D>
__global__ __launch_bounds__(256) void paged_scores_kernel(SplitArgs a)
{
    constexpr int ND = D / 16, NW = 4;
    __shared__ int32_t s_max[NW][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const SplitAt w = split_at(a, blockIdx.x, blockIdx.y, blockIdx.z);
    if (w.t.count == 0 || w.x0 >= w.x1) return;
    int pos;
    v4i qf[D / 64];
    tile_row<D>(a.p, w.t, w.h, c, g, pos, qf);
    int32_t mx = INT32_MIN;
    v4i kf[2][ND];
    auto ask = [&](int x, v4i (&k)[ND]) { load_k<D>(a.p, block_offset<D>(a.p, w.b, w.h, block_at(w.t, x)), lane, k); };
    auto take = [&](int x, const v4i (&k)[ND]) {
        v4i s[4];
        block_scores<D>(a.p, w.t, block_at(w.t, x), pos, g, k, qf, s);
        mx = largest(s, mx);
        if (c < a.held) {
            v4i* dst = reinterpret_cast<v4i*>(a.scores + ((w.index * a.blocks + x) * a.held + c) * 64 + g * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = s[i];
        }
    };
    int x = w.x0 + wave;
    if (x < w.x1) ask(x, kf[0]);
    while (x < w.x1) {
        if (x + NW < w.x1) ask(x + NW, kf[1]);
        take(x, kf[0]);
        x += NW;
        if (x >= w.x1) break;
        if (x + NW < w.x1) ask(x + NW, kf[0]);
        take(x, kf[1]);
        x += NW;
    }
    const auto larger = [](int32_t p, int32_t q) { return p > q ? p : q; };
    mx = combine_rows32(combine_rows16(mx, larger), larger);
    if (g == 0) s_max[wave][c] = mx;
    __syncthreads();
    if (tid < 16) a.maxima[(w.index * a.splits + w.split) * 16 + tid] = larger(larger(s_max[0][tid], s_max[1][tid]), larger(s_max[2][tid], s_max[3][tid]));
}

template <int D>
__global__ __launch_bounds__(256) void paged_values_kernel(SplitArgs a)
{
    constexpr int ND = D / 16, NW = 4;
    __shared__ int32_t s_max[16][17];
    __shared__ int32_t s_hi[D * 16], s_lo[D * 16], s_w[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const SplitAt w = split_at(a, blockIdx.x, blockIdx.y, blockIdx.z);
    if (w.t.count == 0 || w.x0 >= w.x1) return;
    const auto larger = [](int32_t p, int32_t q) { return p > q ? p : q; };
    auto ask = [&](int x, v4i (&v)[ND], v4i (&s)[4]) {
        const v4i* src = reinterpret_cast<const v4i*>(a.scores + ((w.index * a.blocks + x) * a.held + (c < a.held ? c : a.held - 1)) * 64 + g * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = src[i];
        load_v<D>(a.p, block_offset<D>(a.p, w.b, w.h, block_at(w.t, x)), lane, v);
    };
    v4i vf[2][ND], sc[2][4];
    int x = w.x0 + wave;
    if (x < w.x1) ask(x, vf[0], sc[0]);
    // the row's maximum: of all chunks
    {
        const int used = splits_used(a, w.t);
        int32_t m = INT32_MIN;
        for (int i = tid >> 4; i < used; i += 16) m = larger(m, a.maxima[(w.index * a.splits + i) * 16 + (tid & 15)]);
        s_max[tid >> 4][tid & 15] = m;
        for (int i = tid; i < D * 16; i += 256) { s_hi[i] = 0; s_lo[i] = 0; }
        if (tid < 16) s_w[tid] = 0;
    }
    __syncthreads();
    int32_t mx = s_max[0][c];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = larger(mx, s_max[i][c]);

    v4i hi[ND], lo[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) { hi[i] = v4i{0, 0, 0, 0}; lo[i] = v4i{0, 0, 0, 0}; }
    uint32_t sum = 0;
    auto take = [&](const v4i (&v)[ND], const v4i (&s)[4]) {
        v4i wh, wl;
        block_weights(a.p, s, mx, wh, wl, sum);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            hi[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i], wh, hi[i], 0, 0, 0);
            lo[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i], wl, lo[i], 0, 0, 0);
        }
    };
    while (x < w.x1) {
        if (x + NW < w.x1) ask(x + NW, vf[1], sc[1]);
        take(vf[0], sc[0]);
        x += NW;
        if (x >= w.x1) break;
        if (x + NW < w.x1) ask(x + NW, vf[0], sc[0]);
        take(vf[1], sc[1]);
        x += NW;
    }
    // whole numbers: the order of these additions changes nothing
    if (c < a.held) {
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                atomicAdd(&s_hi[c * D + 16 * i + 4 * g + r], hi[i][r]);
                atomicAdd(&s_lo[c * D + 16 * i + 4 * g + r], lo[i][r]);
            }
        atomicAdd(&s_w[c], (int32_t)sum);
    }
    __syncthreads();
    const int64_t at = w.index * a.splits + w.split;
    if (tid < 16) a.sums[at * 16 + tid] = (uint32_t)s_w[tid];
    for (int e = tid; e < a.held * D; e += 256) {
        a.parts[at * a.held * D + e] = (int64_t)s_hi[e] * 256 + s_lo[e];
    }
}

// A workgroup for each row of a tile; its groups of D threads take the chunks in turn, so that all loads are on their way at once (64 chunks of width 128:
// 2 groups 6.4 us, 8 groups 4.7).
constexpr int PJ_THREADS = 1024;
template <int D>
__global__ __launch_bounds__(PJ_THREADS) void paged_join_kernel(SplitArgs a)
{
    constexpr int GROUPS = PJ_THREADS / D;
    __shared__ int64_t s_n[PJ_THREADS];
    __shared__ uint32_t s_w[GROUPS];
    const int tid = threadIdx.x, d = tid % D, part = tid / D, r = blockIdx.x;
    const SplitAt w = split_at(a, 0, blockIdx.y, blockIdx.z);
    if (r >= w.t.count) return;
    const int used = splits_used(a, w.t);
    int64_t N = 0;
    uint32_t W = 0;
#pragma unroll 8
    for (int i = part; i < used; i += GROUPS) {
        const int64_t at = w.index * a.splits + i;
        N += a.parts[(at * a.held + r) * D + d];
        W += a.sums[at * 16 + r];
    }
    s_n[tid] = N;
    if (d == 0) s_w[part] = W;
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) {
        N += s_n[i * D + d];
        W += s_w[i];
    }
    const int f = w.t.first + r, qr = group_of(a.p, f), hd = w.h * a.p.group + (f - qr * a.p.group);
    a.p.out[(int64_t)(w.t.row0 + qr) * a.p.ld_out + hd * D + d] = finished(a.p, N, reciprocal(W));
}

// ---- many rows: prompts ------------------------------------------------------------------------------------------------
// A workgroup of four wavefronts owns 64 rows, a wavefront 16.  First the rows' maxima: a wavefront takes all 64 rows and every fourth
// block of keys, straight from memory into registers (operand order as the cache keeps it), so that no key is read twice and no wavefront
// waits for another before the end.  Then weights and sums, which stay in registers: K and V come a block of 64 keys at a time into
// LDS, one block ahead, for all four.  A weight's two halves are read from a table in LDS, entry DY(m - s): the maximum goes into the
// addend of the score's own 64-bit multiply-add.
// Bound: LDS, and issue next to it.  4096 rows of 32 heads of width 128 (153 us): LDS works 0.58 of the cycles as counted, and some 0.8 of them as a 16-byte read takes 8 where it
// counts 4; 0.24 of the cycles are bank conflicts of the table's reads.  Matrix cores 0.48, vector ALU 0.45.  A score costs a multiply-add, a shift, a cap, an address, a read of 16 bits
// and a permute, and an MFMA takes the place of two and a half vector instructions.  Four wavefronts a SIMD, which is what 16 rows each allow, beat two of 32 rows: those
// read every key from LDS half as often, but two wavefronts issue only every 5.8 cycles.  us, 4096 rows of 32 heads of width 128, 16 rows a wavefront / 32:
// 176 / 194; 32 x 200 rows of 12 heads of width 64 23.0 / 22.6, 4096 of 16 75.8 / 101.
constexpr int PP_TABLE = 1025, PP_NW = 4, PP_ROWS = 64;

// Rows [first, first + n) of a tile, as a tile.
__device__ __forceinline__ Tile part_of(const PagedArgs& a, const Tile& t, int first, int n)
{
    Tile p = t;
    p.first = t.first + first;
    p.count = t.count - first;
    p.count = p.count < 0 ? 0 : (p.count > n ? n : p.count);
    p.low = t.pos0 + group_of(a, p.count > 0 ? p.first : t.first);
    p.high = p.count > 0 ? t.pos0 + group_of(a, p.first + p.count - 1) : -1;
    return p;
}
// The sequence and the tile of PP_ROWS rows that are the index-th of all there are; false: not so many.  A wavefront takes 64 sequences at a time.
__device__ __forceinline__ bool packed_tile(const PagedArgs& a, int32_t index, int& b, int& tile)
{
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < a.packed; b0 += 64) {
        int32_t mine = 0;
        if (b0 + lane < a.packed) {
            const int32_t r0 = clamp_i32(a.q_start[b0 + lane], 0, a.rows), n = clamp_i32(a.q_start[b0 + lane + 1], r0, a.rows) - r0;
            if (!left_out(a, n)) mine = ((n < a.max_q ? n : a.max_q) * a.group + PP_ROWS - 1) / PP_ROWS;
        }
        int32_t sum = mine;
#pragma unroll
        for (int i = 1; i < 64; i *= 2) {
            const int32_t before = __shfl_up(sum, i);
            sum += lane >= i ? before : 0;
        }
        const uint64_t beyond = __builtin_amdgcn_ballot_w64(sum > index);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            b = b0 + at;
            tile = __builtin_amdgcn_readlane(sum, at) - 1 - index;           // (a sequence's last tile, which has most keys, first)
            return true;
        }
        index -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}
// How many of the workgroup's blocks some row of the part may see (the others come last).
__device__ __forceinline__ int blocks_of(const Tile& p)
{
    const int end = (p.high >> 6) + 1;
    return p.high < 0 ? 0 : p.sink_blocks + (end > p.from ? end - p.from : 0);
}
// A lane's row of the part's tile rt: its position and its queries as operand (rows behind the last repeat it).
template <int D>
__device__ __forceinline__ void part_row(const PagedArgs& a, const Tile& p, int h, int rt, int c, int g, int& pos, v4i (&qf)[D / 64])
{
    const int last = p.first + (p.count > 0 ? p.count - 1 : 0);
    int flat = p.first + 16 * rt + c;
    flat = flat < last ? flat : last;
    flat = p.count > 0 ? flat : 0;                         // (a part without rows: the sequence's first, not used)
    const int qi = group_of(a, flat);
    const int8_t* src = a.q + (int64_t)(p.row0 + qi) * a.ld_q + (h * a.group + (flat - qi * a.group)) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) qf[j] = *reinterpret_cast<const v4i*>(src + 64 * j);
    pos = p.pos0 + qi;
}

// Largest raw scores of 64 rows over the blocks first, first + step, ... of the part's: K goes straight from memory into registers, 32 keys while
// the 32 before them are multiplied.
template <int D>
__device__ __forceinline__ void part_maxima(const PagedArgs& a, const Tile& p, int h, int b, int first, int step, int lane, int32_t (&mx)[4])
{
    constexpr int NJ = D / 64, ND = D / 16;
    const auto larger = [](int32_t p, int32_t q) { return p > q ? p : q; };
    const int c = lane & 15, g = lane >> 4, mine = blocks_of(p);
    int pos[4];
    v4i qf[4][NJ];
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) {
        part_row<D>(a, p, h, rt, c, g, pos[rt], qf[rt]);
        mx[rt] = INT32_MIN;
    }
    v4i k0[ND / 2], k1[ND / 2];
    auto ask = [&](int64_t at, v4i (&k)[ND / 2]) {
#pragma unroll
        for (int i = 0; i < ND / 2; ++i) k[i] = *reinterpret_cast<const v4i*>(a.k + at + i * 1024 + lane * 16);
    };
    // (a block that all rows see whole in one run of code, without tests between its matrix instructions)
    auto scores = [&](int i, const v4i (&k)[ND / 2], v4i (&s)[4]) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) s[rt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[i * NJ + j], qf[rt][j], j == 0 ? v4i{0, 0, 0, 0} : s[rt], 0, 0, 0);
    };
    auto compare = [&](const v4i (&s)[4]) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx[rt] = larger(mx[rt], s[rt][r]);
    };
    auto take = [&](int key, bool whole, const v4i (&k)[ND / 2]) {
        if (whole) {
            v4i s[2][4];
            scores(0, k, s[0]);
            scores(1, k, s[1]);
            compare(s[0]);
            compare(s[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v4i s[4];
                scores(i, k, s);
#pragma unroll
                for (int rt = 0; rt < 4; ++rt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!visible(a, key + 16 * i + 4 * g + r, pos[rt])) s[rt][r] = INT32_MIN;
                compare(s);
            }
        }
    };
    if (first < mine) ask(block_offset<D>(a, b, h, block_at(p, first)), k0);
    for (int x = first; x < mine; x += step) {
        const int block = block_at(p, x);
        const bool whole = whole_block(a, p, block);
        ask(block_offset<D>(a, b, h, block) + 32 * D, k1);
        take(64 * block, whole, k0);
        ask(block_offset<D>(a, b, h, block_at(p, x + step < mine ? x + step : x)), k0);
        take(64 * block + 32, whole, k1);
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) mx[rt] = combine_rows32(combine_rows16(mx[rt], larger), larger);
}

template <int D, bool HIGH>
__global__ __launch_bounds__(64 * PP_NW, 4) void paged_prompt_kernel(PagedArgs a)
{
    constexpr int NJ = D / 64, ND = D / 16, BLOCK = 64 * D, NW = PP_NW;
    __shared__ __attribute__((aligned(16))) int8_t blocks[4][BLOCK];          // K twice, V twice
    __shared__ uint16_t table[PP_TABLE];
    __shared__ int32_t maxima[NW][PP_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int h = blockIdx.x;
    int b = blockIdx.z, tile = gridDim.y - 1 - blockIdx.y;                   // (the rows with most keys first)
    if (a.packed && !packed_tile(a, blockIdx.y, b, tile)) return;
    const Tile t = tile_of(a, b, tile, PP_ROWS);
    if (t.count == 0) return;
    const int n = t.blocks;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t*)&blocks[0][0];
    auto offset = [&](int x) { return block_offset<D>(a, b, h, block_at(t, x < n ? x : (n > 0 ? n - 1 : 0))); };
    auto request = [&](int64_t at, int buffer) {
#pragma unroll
        for (int i = 0; i < 2 * ND / NW; ++i) {
            const int piece = NW * i + wave;               // K's pieces of 1 KB, then V's
            const bool of_v = piece >= ND;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                         :: "s"(lds0 + (uint32_t)((of_v ? 2 * BLOCK - ND * 1024 : 0) + buffer * BLOCK + piece * 1024)),
                            "v"((uint32_t)((piece - (of_v ? ND : 0)) * 1024 + lane * 16)), "s"((of_v ? a.v : a.k) + at) : "memory", "m0");
        }
    };
    if (n > 0) request(offset(0), 0);
    for (int e = tid; e < PP_TABLE; e += 64 * NW) {
        const uint32_t z = (uint32_t)e >> 6, f = 124u - (e & 63u);
        const uint32_t w = (umad24(f, f, 8180u) + ((1u << z) >> 1)) >> z;
        table[e] = (uint16_t)((w & 255u) | ((w + 128u) >> 8 << 8));
    }

    // ---- maxima -------------------------------------------------------------------------------------------------
    {
        int32_t mx[4];
        part_maxima<D>(a, t, h, b, wave, NW, lane, mx);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
            if (g == 0) maxima[wave][16 * rt + c] = mx[rt];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");          // (and the table is made)

    // ---- weights and sums ----------------------------------------------------------------------------------------
    const Tile own = part_of(a, t, wave * 16, 16);
    const int mine = blocks_of(own);
    int pos;
    v4i qf[NJ], hi[ND], lo[ND];
    part_row<D>(a, own, h, 0, c, g, pos, qf);
    int32_t mx = INT32_MIN;
    v4i sum_h{0, 0, 0, 0}, sum_l{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < NW; ++i) mx = mx > maxima[i][wave * 16 + c] ? mx : maxima[i][wave * 16 + c];
#pragma unroll
    for (int i = 0; i < ND; ++i) { hi[i] = v4i{0, 0, 0, 0}; lo[i] = v4i{0, 0, 0, 0}; }
    // DY(m - s) = (s * -factor + (m * factor + 2^(shift-1))) >> shift
    const int32_t minus_m = -(int32_t)a.s_m;
    const v4i ones = {0x01010101, 0x01010101, 0x01010101, 0x01010101};
    const int64_t row_c = (int64_t)mx * (int32_t)a.s_m + ((int64_t)1 << (HIGH ? a.s_s + 31 : a.s_s - 1));
    for (int x = 0; x < n; ++x) {
        const int64_t next = offset(x + 1);
        // block x has landed, for everybody, and everybody has left block x - 1
        __builtin_amdgcn_s_waitcnt(0x0070);
        asm volatile("s_barrier" ::: "memory");
        request(next, (x + 1) & 1);                        // (behind the last block: that one again)
        if (x >= mine) continue;
        const int block = block_at(t, x);
        v4i s[4], wh, wl;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const v4i kf = *reinterpret_cast<const v4i*>(&blocks[x & 1][(i * NJ + j) * 1024 + lane * 16]);
                s[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf, qf[j], j == 0 ? v4i{0, 0, 0, 0} : s[i], 0, 0, 0);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t p = (int64_t)s[i][r] * minus_m + row_c;
                const uint32_t d = HIGH ? (uint32_t)(p >> 32) >> (a.s_s & 31) : __builtin_amdgcn_alignbit((uint32_t)(p >> 32), (uint32_t)p, (uint32_t)(a.s_s & 31));
                s[i][r] = (int32_t)(d < PP_TABLE - 1u ? d : PP_TABLE - 1u);
            }
        if (!whole_block(a, own, block)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!visible(a, 64 * block + 16 * i + 4 * g + r, pos)) s[i][r] = PP_TABLE - 1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[i][r] = table[s[i][r]];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = __builtin_amdgcn_perm((uint32_t)s[i][1], (uint32_t)s[i][0], 0x05010400u);
            const uint32_t q = __builtin_amdgcn_perm((uint32_t)s[i][3], (uint32_t)s[i][2], 0x05010400u);
            wl[i] = (int32_t)__builtin_amdgcn_perm(q, p, 0x05040100u);
            wh[i] = (int32_t)__builtin_amdgcn_perm(q, p, 0x07060302u);
        }
        // sums of the weights, as the product with a value of 1 (eight dot instructions otherwise: 1 % of a long prompt)
        sum_h = __builtin_amdgcn_mfma_i32_16x16x64_i8(ones, wh, sum_h, 0, 0, 0);
        sum_l = __builtin_amdgcn_mfma_i32_16x16x64_i8(ones, wl, sum_l, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const v4i vf = *reinterpret_cast<const v4i*>(&blocks[2 + (x & 1)][i * 1024 + lane * 16]);
            hi[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf, wh, hi[i], 0, 0, 0);
            lo[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf, wl, lo[i], 0, 0, 0);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                    // (nothing is on its way into LDS any more)
    if (c >= own.count) return;
    const uint64_t R = reciprocal(((uint32_t)sum_h[0] << 8) + (uint32_t)sum_l[0]);
    const int flat = own.first + c, qi = group_of(a, flat);
    int8_t* dst = a.out + (int64_t)(t.row0 + qi) * a.ld_out + (h * a.group + (flat - qi * a.group)) * D + 4 * g;
#pragma unroll
    for (int i = 0; i < ND; ++i) {
        int32_t y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = finished(a, (int64_t)hi[i][r] * 256 + lo[i][r], R);
        *reinterpret_cast<uint32_t*>(dst + 16 * i) = pack4_perm(y[0], y[1], y[2], y[3]);
    }
}

static int g_paged_form = -1;          // see ibert_paged_attention_override

// Which kernels run, and their workspace.
struct Plan {
    int32_t prompt_tiles, high;                     // > 0: paged_prompt_kernel; the scores' shift is 32 or more
    int32_t room;                                   // > 0: paged_row_kernel, with so many blocks of scores
    int32_t tiles, splits, chunk, blocks, held;     // chunk > 0: the three kernels for few rows
    size_t maxima, sums, parts, scores, total;      // bytes from the workspace's start
};
static Plan plan_paged(const ibert_paged_attention_desc& d, const ibert_kv_cache& c, int32_t batch, int32_t max_q_len, int32_t max_kv_len)
{
    Plan p = {};
    const int64_t rows = (int64_t)max_q_len * (d.heads_q / c.heads_kv);
    int64_t blocks = max_kv_len > 0 ? ((int64_t)max_kv_len + 63) / 64 : 1;
    if (d.window > 0) {
        const int64_t seen = ((int64_t)d.sinks + 63) / 64 + ((int64_t)d.window + max_q_len + 62) / 64 + 1;
        blocks = blocks < seen ? blocks : seen;
    }
    p.tiles = (int32_t)((rows + 15) / 16);
    p.held = rows < 16 ? (int32_t)rows : 16;
    p.splits = 1;
    p.high = d.scores_dy.s >= 32;
    const int form = g_paged_form;
    const int64_t prompt_tiles = (rows + PP_ROWS - 1) / PP_ROWS;
    const int64_t seqs = (int64_t)batch * c.heads_kv, problems = seqs * p.tiles;
    // Prompts: a workgroup of the prompt kernel takes four times the rows, so it wants more of them before the chip is full, and most of their rows filled.  us,
    // the scores made twice / this, 8 key heads of width 128 with 4 queries each: 1 x 300 rows on 8000 keys (152 workgroups) 99 / 135, 1 x 512 (256) 20.7 / 18.5, on
    // 8000 keys 136 / 140, 1 x 1024 (512) 39.6 / 29.4, on 8000 keys 245 / 168; 16 heads of width 64: 2 x 512 (256) 12.5 / 14.7, 1 x 2048 (512) 38.4 / 36.4; 12:
    // 8 x 200 (384) 11.3 / 11.9, 32 x 200 (1536) 30.4 / 23.3.  Few rows each, by 16-row tiles: width 128, 40 x 5 (640) on 600 keys 18.8 / 21.3, on 1500 42.1 / 40.5, on
    // 4000 111 / 98, 40 x 12 (960) on 600 27.1 / 22.4; width 64, 30 x 20 (720) on 1000 17.5 / 21.7, on 4000 60 / 66, 30 x 40 (1080) on 1000 23.5 / 22.4, on 4000 87 / 69.
    const bool many = prompt_tiles * seqs >= 320 && problems >= (c.head_dim == 128 && blocks >= 24 ? 640 : 960);
    if (p.tiles > 65535 || (form < 0 ? rows > 16 && many : form == IBERT_PAGED_PROMPT)) {
        p.prompt_tiles = (int32_t)prompt_tiles;
        return p;
    }
    if (batch == 0) return p;
    // One launch where the scores of all keys fit LDS, unless that leaves few workgroups with long ways: a workgroup takes some 0.2 us a block and the three
    // launches 12 and more.  us, three launches / one, of 8 key heads of width 128, 4 rows: 1 x 1000 keys 11.9 / 9.9, 1 x 2000 12.4 / 13.4, 1 x 4000 12.9 / 20.1,
    // 8 x 4000 22.3 / 22.3, 16 x 1500 18.6 / 13.4, 24 x 4000 44.0 / 32.1, 64 x 4096 94.6 / 71.6; 12 of width 64, 1 row: 4 x 2000 12.8 / 11.2, 2 x 4000 13.5 / 18.2.
    const int64_t lds = (int64_t)p.held * (256 * blocks + 8 * c.head_dim);
    if (lds <= 128 * 1024 && (form < 0 ? rows <= 16 && (blocks <= 24 || problems >= 64) : form == IBERT_PAGED_ONE)) {
        p.room = (int32_t)blocks;
        return p;
    }
    int64_t splits = (512 + problems - 1) / problems;
    int64_t chunk = (blocks + splits - 1) / splits;
    if (chunk < 4) chunk = 4;
    splits = (blocks + chunk - 1) / chunk;
    // Keys split where a workgroup's way along them takes longer than two more launches and what they hand on.  Both are estimated, in ns, with the bounds that the host
    // knows: 0.27 us a block (width 64 0.23) or the bytes of K twice and V; 11 us, the bytes of K and V, and those of the scores and partial sums.  us, twice / split,
    // blocks of keys x tiles, width 128: 4 rows a tile 47 x 8 17.0 / 12.3, 47 x 128 20.8 / 24.4, 188 x 128 88 / 70, 188 x 320 208 / 190; 8 rows 188 x 32 69 / 35, 47 x 128
    // 27 / 38; 16 rows 63 x 16 21.9 / 19.2, 63 x 32 22 / 27, 188 x 32 69 / 46, 188 x 128 110 / 135, 938 x 16 310 / 67; width 64, 1 row 125 x 48 31.8 / 20.0, 12 rows
    // 125 x 12 32 / 18, 125 x 48 33 / 33, 125 x 144 41 / 75.
    const int64_t block_bytes = seqs * blocks * 64 * c.head_dim, along = blocks * (c.head_dim == 128 ? 270 : 230), thrice = block_bytes * 3 / 4600;
    const int64_t handed_on = problems * p.held * (blocks * 512 + splits * c.head_dim * 16);
    if (form < 0 ? 6000 + (along > thrice ? along : thrice) <= 11000 + block_bytes * 2 / 5000 + handed_on / 3000 : form != IBERT_PAGED_SPLIT) return p;
    p.splits = (int32_t)splits; p.chunk = (int32_t)chunk; p.blocks = (int32_t)blocks;
    const auto room = [&](int64_t n) {
        const size_t at = p.total;
        p.total += (size_t)((n + 255) / 256 * 256);
        return at;
    };
    p.maxima = room(problems * splits * 64);
    p.sums = room(problems * splits * 64);
    p.parts = room(problems * splits * p.held * c.head_dim * 8);
    p.scores = room(problems * blocks * p.held * 256);
    if (p.total > ((size_t)2 << 30)) { p.total = 0; p.chunk = 0; }      // (not for so much room: the scores are made twice then)
    return p;
}

// Single rows among prompts (a step of a server): the prompt kernel walks a single row's keys with one workgroup a key head.  Where the others have a sixteenth of the
// longest's rows on average, sequences of one row go by a plan of their own, and the prompt kernel leaves them out.  us, together / apart, 8 key heads of width 128 with 4
// queries each, single rows on 2000 keys and a prompt: 63 and 512 rows 110 / 62, 15 and 512 50 / 34, 63 (4000 keys) and 2048 272 / 157, 1 (60000 keys) and 1024 755 / 59.  Not
// where prompts are short or many: 15 rows on 500 keys and 40 rows 18 / 23, 180 on 800 and 20 prompts of 100 115 / 138, 8 of 8 to 500 rows 19 / 21.
static bool is_mixed(const ibert_paged_attention_desc& d, const ibert_kv_cache& c, const Plan& plan, int32_t batch, int32_t rows, int32_t max_q_len)
{
    return g_paged_form < 0 && plan.prompt_tiles > 0 && batch > 1 && (int64_t)max_q_len * (d.heads_q / c.heads_kv) >= 512 &&
           (int64_t)rows - max_q_len <= (int64_t)(batch - 1) * max_q_len / 16;
}

template <int D>
static int launch_paged(PagedArgs a, const Plan& plan, int32_t batch, void* workspace, hipStream_t stream)
{
    if (plan.prompt_tiles > 0) {
        // At most so many tiles have rows.  Where the grid would be four times that, tiles are counted instead: a workgroup without rows costs some 0.5 ns, and 64 x 2048 rows
        // of which 2111 are there, 190 us with them, 157 without.
        const int64_t filled = (int64_t)a.rows * a.group / PP_ROWS + (batch < a.rows ? batch : a.rows);
        a.packed = a.q_start && filled <= 65535 && 4 * filled <= (int64_t)batch * plan.prompt_tiles ? batch : 0;
        const dim3 grid((unsigned)a.heads_kv, (unsigned)(a.packed ? filled : plan.prompt_tiles), (unsigned)(a.packed ? 1 : batch)), block(64 * PP_NW);
        if (plan.high) hipLaunchKernelGGL((paged_prompt_kernel<D, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((paged_prompt_kernel<D, false>), grid, block, 0, stream, a);
        IBERT_LAUNCH_CHECK("paged_prompt_kernel");
        g_last_kernel = "paged_prompt_kernel";
        return IBERT_OK;
    }
    if (plan.room > 0) {
        const size_t lds = (size_t)plan.held * (256 * plan.room + 8 * D);
        auto kern = paged_row_kernel<D>;
        if (lds > 60000)
            IBERT_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 132 * 1024));
        hipLaunchKernelGGL(kern, dim3((unsigned)a.heads_kv, (unsigned)batch, (unsigned)plan.tiles), dim3(64 * PW_NW), lds, stream, a, plan.held, plan.room);
        IBERT_LAUNCH_CHECK("paged_row_kernel");
        g_last_kernel = "paged_row_kernel";
        return IBERT_OK;
    }
    if (plan.chunk == 0) {
        const dim3 grid((unsigned)a.heads_kv, (unsigned)batch, (unsigned)plan.tiles);
        if ((int64_t)a.heads_kv * batch * plan.tiles <= 256) hipLaunchKernelGGL((paged_attention_kernel<D, 8>), grid, dim3(512), 0, stream, a);
        else hipLaunchKernelGGL((paged_attention_kernel<D, 4>), grid, dim3(256), 0, stream, a);
        IBERT_LAUNCH_CHECK("paged_attention_kernel");
        g_last_kernel = "paged_attention_kernel";
        return IBERT_OK;
    }
    SplitArgs s;
    s.p = a; s.tiles = plan.tiles; s.splits = plan.splits; s.chunk = plan.chunk; s.blocks = plan.blocks; s.held = plan.held;
    char* ws = static_cast<char*>(workspace);
    s.maxima = reinterpret_cast<int32_t*>(ws + plan.maxima); s.sums = reinterpret_cast<uint32_t*>(ws + plan.sums);
    s.parts = reinterpret_cast<int64_t*>(ws + plan.parts); s.scores = reinterpret_cast<int32_t*>(ws + plan.scores);
    const dim3 grid((unsigned)plan.splits, (unsigned)(a.heads_kv * plan.tiles), (unsigned)batch);
    hipLaunchKernelGGL(paged_scores_kernel<D>, grid, dim3(256), 0, stream, s);
    IBERT_LAUNCH_CHECK("paged_scores_kernel");
    hipLaunchKernelGGL(paged_values_kernel<D>, grid, dim3(256), 0, stream, s);
    IBERT_LAUNCH_CHECK("paged_values_kernel");
    hipLaunchKernelGGL(paged_join_kernel<D>, dim3((unsigned)plan.held, grid.y, grid.z), dim3(PJ_THREADS), 0, stream, s);
    IBERT_LAUNCH_CHECK("paged_join_kernel");
    g_last_kernel = "paged_join_kernel";
    return IBERT_OK;
}

static int check_paged(const ibert_paged_attention_desc* desc, const ibert_kv_cache* cache, int32_t batch, int32_t rows, int32_t max_q_len, int32_t max_kv_len)
{
    if (!desc || !cache) return IBERT_ERR_NULL;
    if (const int rc = check_cache(cache)) return rc;
    const ibert_paged_attention_desc& d = *desc;
    if (batch < 0 || batch > 65535 || rows < 0 || max_q_len < 1 || max_kv_len < 0 || d.heads_q < 1 || d.heads_q > (1 << 20) || d.heads_q % cache->heads_kv ||
        (int64_t)max_q_len * (d.heads_q / cache->heads_kv) > 65535 * 64) return IBERT_ERR_SHAPE;
    if (max_kv_len > PA_MOST_KEYS || d.scores_dy.m < 0 || d.scores_dy.s < 24 || d.scores_dy.s > 62 || !dyadic_ok(d.out_dy) || d.window < 0 || d.sinks < 0)
        return IBERT_ERR_PARAM_RANGE;
    return IBERT_OK;
}

}  // namespace ibert

extern "C" void ibert_paged_attention_override(int32_t form) { ibert::g_paged_form = form; }

extern "C" size_t ibert_paged_attention_workspace_bytes(const ibert_paged_attention_desc* desc, const ibert_kv_cache* cache, int32_t batch,
                                                        int32_t rows, int32_t max_q_len, int32_t max_kv_len)
{
    if (ibert::check_paged(desc, cache, batch, rows, max_q_len, max_kv_len)) return 0;
    const ibert::Plan plan = ibert::plan_paged(*desc, *cache, batch, max_q_len, max_kv_len);
    if (ibert::is_mixed(*desc, *cache, plan, batch, rows, max_q_len)) return ibert::plan_paged(*desc, *cache, batch, 1, max_kv_len).total;
    return plan.total;
}

extern "C" int ibert_paged_attention_i(const ibert_paged_attention_desc* desc, const ibert_kv_cache* cache, const int8_t* q, int64_t ld_q,
                                       const int32_t* block_table, int32_t max_pages, const int32_t* q_start, const int32_t* kv_len,
                                       int32_t batch, int32_t rows, int32_t max_q_len, int32_t max_kv_len, int8_t* out, int64_t ld_out,
                                       void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace ibert;
    if (const int rc = check_paged(desc, cache, batch, rows, max_q_len, max_kv_len)) return rc;
    const ibert_paged_attention_desc& d = *desc;
    const int D = cache->head_dim;
    if (max_pages < 1 || ld_q < (int64_t)d.heads_q * D || ld_out < (int64_t)d.heads_q * D || (!q_start && rows < batch)) return IBERT_ERR_SHAPE;
    if (batch == 0 || rows == 0) return IBERT_OK;
    if (!q || !out || !block_table || !kv_len || !cache->k || !cache->v) return IBERT_ERR_NULL;
    if (!aligned(q, 16) || ld_q % 16 || !aligned(out, 4) || ld_out % 4 || !aligned(cache->k, 16) || !aligned(cache->v, 16)) return IBERT_ERR_ALIGN;
    const Plan prompts = plan_paged(d, *cache, batch, max_q_len, max_kv_len);
    const bool mixed = is_mixed(d, *cache, prompts, batch, rows, max_q_len);
    const Plan plan = mixed ? plan_paged(d, *cache, batch, 1, max_kv_len) : prompts;
    if (plan.total > 0 && (!workspace || workspace_bytes < plan.total || !aligned(workspace, 256))) return IBERT_ERR_WORKSPACE;
    PagedArgs a;
    a.q = q; a.k = cache->k; a.v = cache->v; a.out = out; a.table = block_table; a.q_start = q_start; a.kv_len = kv_len;
    a.ld_q = ld_q; a.ld_out = ld_out; a.heads_q = d.heads_q; a.heads_kv = cache->heads_kv; a.group = d.heads_q / cache->heads_kv;
    a.group_magic = udiv_magic(a.group);
    a.log_page = __builtin_ctz((unsigned)cache->page_size); a.num_pages = cache->num_pages; a.max_pages = max_pages; a.rows = rows; a.max_q = max_q_len;
    const int64_t held = (int64_t)max_pages << a.log_page;
    a.keys = (int32_t)(held < max_kv_len ? held : max_kv_len);
    // (a window of all keys there can be is none, and so many first tokens are all)
    a.window = d.window >= PA_MOST_KEYS ? 0 : d.window; a.sinks = d.sinks < PA_MOST_KEYS ? d.sinks : PA_MOST_KEYS;
    const int s = d.scores_dy.s;
    a.s_m = (uint32_t)d.scores_dy.m; a.s_l = s < 32 ? 32 - s : 0; a.s_r = s > 32 ? s - 32 : 0; a.s_rnd = (uint64_t)1 << (s < 32 ? 31 : s - 1);
    a.s_s = s >= 32 ? s - 32 : s;
    a.out_dy = d.out_dy; a.only = mixed;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const auto launch = [&](const Plan& p) { return D == 64 ? launch_paged<64>(a, p, batch, workspace, st) : launch_paged<128>(a, p, batch, workspace, st); };
    const int rc = launch(plan);
    if (rc || !mixed) return rc;
    a.only = 2;
    return launch(prompts);
}
