// Block tables and slot maps of a paged key/value cache from request lengths (ibert_page_tables_i).
//
// Everything a step needs follows from three running sums over the batch: pages taken, pages put back, rows given out.  They
// are a few thousand integers, so every workgroup makes all of them for itself in LDS (two passes: what is asked for decides
// what is granted) and then writes its share of the rows and of the pages, each of which finds its sequence by bisection of
// those sums.  One launch, no workspace, nothing passed between workgroups; the order of the pages is that of the sequences.
// Bound: latency (a launch, two dependent trips to memory, the sums): a batch of one 2.9 us, 512 sequences of up to 8192 tokens with prompts among them 5.3
// (kernel trace), where an empty kernel takes 2.2.  Passing the sums from one workgroup to the others would be a second launch or a wait.
#include "common.h"

namespace ibert {

constexpr int PT_THREADS = 512, PT_WAVES = PT_THREADS / 64, PT_MOST = 8192;

struct PageArgs {
    const int32_t *before, *after, *ring_in;
    int32_t *ring, *ring_out, *table, *q_start, *kv_len, *slots, *positions;
    int32_t batch, log_page, num_pages, max_pages, rows;
};

// Sums of what is asked for may pass 32 bits: they stop at 2^32 - 1, above everything they are compared with (rows and pages,
// at most 2^31 - 1).  (Addition that stops there is associative, so a scan may group it as it likes.)
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// The value some lanes before this one in its row of 16 (or the last of the rows before it), 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_before(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int32_t)v, CTRL, ROWS, 0xF, false);
}

// Inclusive sums of N values over the workgroup; total[] = those of all threads.  tmp: PT_WAVES * N words.
template <int N, bool SAT>
__device__ __forceinline__ void block_scan(uint32_t (&v)[N], uint32_t (&total)[N], uint32_t* tmp)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto add = [](uint32_t a, uint32_t b) { return SAT ? add_sat(a, b) : a + b; };
#pragma unroll
    for (int n = 0; n < N; ++n) {
        v[n] = add(v[n], dpp_before<0x111, 0xF>(v[n]));    // row_shr 1, 2, 4, 8
        v[n] = add(v[n], dpp_before<0x112, 0xF>(v[n]));
        v[n] = add(v[n], dpp_before<0x114, 0xF>(v[n]));
        v[n] = add(v[n], dpp_before<0x118, 0xF>(v[n]));
        v[n] = add(v[n], dpp_before<0x142, 0xA>(v[n]));    // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
        v[n] = add(v[n], dpp_before<0x143, 0xC>(v[n]));
    }
    __syncthreads();                                       // (tmp may still be read from an earlier call)
    if (lane == 63)
#pragma unroll
        for (int n = 0; n < N; ++n) tmp[wave * N + n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        uint32_t before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < PT_WAVES; ++w) {
            const uint32_t t = tmp[w * N + n];
            if (w == wave) before = all;
            all = add(all, t);
        }
        v[n] = add(v[n], before);
        total[n] = all;
    }
}

// First index whose entry is above x, of n ascending entries.
__device__ __forceinline__ int above(const uint32_t* ends, int n, uint32_t x)
{
    int lo = 0, hi = n - 1;                                // (the caller knows that the last one is)
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__global__ __launch_bounds__(PT_THREADS) void page_tables_kernel(PageArgs a)
{
    extern __shared__ uint32_t pt_lds[];
    __shared__ uint32_t tmp[PT_WAVES * 4];
    uint32_t* const row_end = pt_lds;                      // running sums of what is granted: rows, pages taken, pages put back
    uint32_t* const take_end = row_end + a.batch;
    uint32_t* const back_end = take_end + a.batch;
    int32_t* const before_of = reinterpret_cast<int32_t*>(back_end + a.batch);
    const int tid = threadIdx.x, lp = a.log_page;
    const uint32_t R = (uint32_t)a.num_pages;
    int32_t head = a.ring_in[0], count = a.ring_in[1];
    head = clamp_i32(head, 0, a.num_pages - 1);
    count = clamp_i32(count, 0, a.num_pages);
    const auto pages = [&](int32_t len) { return (uint32_t)(((uint32_t)len + (1u << lp) - 1u) >> lp); };

    uint32_t asked[2] = {0, 0}, given[4] = {0, 0, 0, 0};  // sums before the chunk
    for (int b0 = 0; b0 < a.batch; b0 += PT_THREADS) {
        const int b = b0 + tid;
        const bool in = b < a.batch;
        int32_t before = in ? a.before[b] : 0, after = in ? a.after[b] : 0;
        before = before < 0 ? 0 : before;
        after = after < 0 ? 0 : after;
        const uint32_t had = pages(before), wants = pages(after);
        const uint32_t need = wants > had ? wants - had : 0, rows = after > before ? (uint32_t)(after - before) : 0;
        uint32_t v[2] = {need, rows}, all[2];
        block_scan<2, true>(v, all, tmp);
        const bool granted = wants <= (uint32_t)a.max_pages && (need == 0 || add_sat(asked[0], v[0]) <= (uint32_t)count) &&
                             (rows == 0 || add_sat(asked[1], v[1]) <= (uint32_t)a.rows);
        asked[0] = add_sat(asked[0], all[0]);
        asked[1] = add_sat(asked[1], all[1]);
        // (a sequence never puts back more pages than its row of the table names)
        const uint32_t held = had < (uint32_t)a.max_pages ? had : (uint32_t)a.max_pages;
        uint32_t g[4] = {granted ? rows : 0, granted ? need : 0, granted && held > wants ? held - wants : 0, in && !granted}, sum[4];
        block_scan<4, false>(g, sum, tmp);
        if (in) {
            before_of[b] = before;
            row_end[b] = given[0] + g[0];
            take_end[b] = given[1] + g[1];
            back_end[b] = given[2] + g[2];
            if (blockIdx.x == 0) {
                a.kv_len[b] = granted ? after : before;
                a.q_start[b + 1] = (int32_t)(given[0] + g[0]);
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) given[n] += sum[n];
    }
    const uint32_t rows = given[0], taken = given[1], back = given[2];
    if (blockIdx.x == 0 && tid == 0) {
        a.q_start[0] = 0;
        a.ring_out[0] = (int32_t)(((uint32_t)head + taken) % R);
        const uint32_t left = (uint32_t)count - taken + back;
        a.ring_out[1] = (int32_t)(left < R ? left : R);
        a.ring_out[2] = (int32_t)given[3];
    }
    __syncthreads();

    const uint32_t first = blockIdx.x * PT_THREADS + tid, step = gridDim.x * PT_THREADS;
    const auto length = [&](int b) { return before_of[b]; };
    // the i-th page that is taken
    const auto page_of = [&](uint32_t i) {                 // (i < count <= R)
        const uint32_t k = (uint32_t)head + i;
        return a.ring[k < R ? k : k - R];
    };
    for (uint32_t i = first; i < taken; i += step) {
        const int b = above(take_end, a.batch, i);
        const uint32_t p = pages(length(b)) + i - (b ? take_end[b - 1] : 0);
        a.table[(int64_t)b * a.max_pages + p] = page_of(i);
    }
    for (uint32_t i = first; i < back; i += step) {
        const int b = above(back_end, a.batch, i);
        const uint32_t had = pages(length(b)), held = had < (uint32_t)a.max_pages ? had : (uint32_t)a.max_pages;
        a.ring[((uint32_t)head + (uint32_t)count + i) % R] = a.table[(int64_t)b * a.max_pages + (held - (back_end[b] - i))];
    }
    for (uint32_t t = first; t < (uint32_t)a.rows; t += step) {
        int32_t slot = -1, pos = 0;
        if (t < rows) {
            const int b = above(row_end, a.batch, t);
            const int32_t before = length(b);
            pos = before + (int32_t)(t - (b ? row_end[b - 1] : 0));
            const uint32_t p = (uint32_t)pos >> lp, had = pages(before);
            const int32_t page = p < had ? a.table[(int64_t)b * a.max_pages + p] : page_of((b ? take_end[b - 1] : 0) + p - had);
            slot = (int32_t)(((uint32_t)page << lp) + ((uint32_t)pos & ((1u << lp) - 1u)));
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
}

static int launch_page_tables(const PageArgs& a, hipStream_t stream)
{
    // a thread for every row, as long as a workgroup has 512 to do
    const int64_t wgs = ((int64_t)a.rows + PT_THREADS - 1) / PT_THREADS;
    const size_t lds = 16 * (size_t)a.batch;
    auto kern = page_tables_kernel;
    if (lds > 60000)
        IBERT_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 16 * PT_MOST));
    hipLaunchKernelGGL(kern, dim3((unsigned)(wgs < 1 ? 1 : (wgs > 256 ? 256 : wgs))), dim3(PT_THREADS), lds, stream, a);
    IBERT_LAUNCH_CHECK("page_tables_kernel");
    g_last_kernel = "page_tables_kernel";
    return IBERT_OK;
}

}  // namespace ibert

extern "C" int ibert_page_tables_i(const int32_t* len_before, const int32_t* len_after, int32_t batch, int32_t page_size,
                                   int32_t num_pages, const int32_t* ring_in, int32_t* free_ring, int32_t* ring_out,
                                   int32_t* block_table, int32_t max_pages, int32_t rows, int32_t* q_start, int32_t* kv_len,
                                   int32_t* slots, int32_t* positions, void* stream)
{
    if (batch < 0 || batch > ibert::PT_MOST || page_size < 64 || (page_size & (page_size - 1)) || num_pages < 1 || max_pages < 1 || rows < 0 ||
        (int64_t)num_pages * page_size > 0x7fffffffLL || (int64_t)max_pages * page_size > 0x7fffffffLL ||
        (int64_t)batch * max_pages > 0x7fffffffLL) return IBERT_ERR_SHAPE;
    if (!ring_in || !free_ring || !ring_out || !q_start) return IBERT_ERR_NULL;
    if (batch > 0 && (!len_before || !len_after || !block_table || !kv_len)) return IBERT_ERR_NULL;
    if (rows > 0 && (!slots || !positions)) return IBERT_ERR_NULL;
    // (workgroups read what the inputs were while others write: no written array may share a word with another)
    const int64_t n = batch, r = rows;
    const struct { const int32_t* p; int64_t words; } arrays[] = {
        {free_ring, num_pages}, {ring_out, 3}, {block_table, n * max_pages}, {q_start, n + 1}, {kv_len, n}, {slots, r}, {positions, r},        // written
        {len_before, n}, {len_after, n}, {ring_in, 2}};
    for (int w = 0; w < 7; ++w)
        for (int o = w + 1; o < 10; ++o) {
            const auto &x = arrays[w], &y = arrays[o];
            const uintptr_t px = reinterpret_cast<uintptr_t>(x.p), py = reinterpret_cast<uintptr_t>(y.p);
            if (x.words > 0 && y.words > 0 && px < py + 4 * (uint64_t)y.words && py < px + 4 * (uint64_t)x.words) return IBERT_ERR_SHAPE;
        }
    ibert::PageArgs a;
    a.before = len_before; a.after = len_after; a.ring_in = ring_in;
    a.ring = free_ring; a.ring_out = ring_out; a.table = block_table; a.q_start = q_start; a.kv_len = kv_len; a.slots = slots; a.positions = positions;
    a.batch = batch; a.log_page = __builtin_ctz((unsigned)page_size); a.num_pages = num_pages; a.max_pages = max_pages; a.rows = rows;
    return ibert::launch_page_tables(a, static_cast<hipStream_t>(stream));
}
