// page_kernels.hip -- the paged 8-bit cache, for gfx950: block tables and slot
// maps from request lengths, and the writing and reading back of K/V rows.
#include "page_rows_device.h"

namespace fkv {
namespace {

constexpr int kThreads = 256;

// --------------------------------------------------------------------- plan --

// Sums that stop at 2^31 - 1: of any lengths, in 32 bits, and in any order.
constexpr uint32_t kSumMost = 0x7fffffffu;

__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return min(a + b, kSumMost); }

// Sum over the threads before this one of a block's 256, and over all; `part`
// holds a word per wave.  Ends with a barrier, so `part` may be used again.
__device__ __forceinline__ uint32_t block_sum_before(uint32_t v, uint32_t* part, uint32_t& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const uint32_t u = __shfl_up(v, k, 64);
        if (lane >= k) v = plus(v, u);
    }
    if (lane == 63) part[wave] = v;
    uint32_t before = __shfl_up(v, 1, 64);
    if (lane == 0) before = 0;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before = plus(before, part[w]);
        total = plus(total, part[w]);
    }
    __syncthreads();
    return before;
}

// Two prefix sums over the requests, of their rows and of the pages that they
// need, say where each row and each further page of every request goes; all
// else is a gather.  Both sums are cheap beside a second launch and a pass of
// the sums through memory, so every block forms them for itself, kPlanTile
// requests at a time in LDS, and writes its share of the rows and pages:
// kThreads consecutive ones at a time, the blocks taking turns, kPlanTurns
// turns' look-ups in flight at once.  A wave finds the request of its first row
// by two 64-way probes of the sums, and the others mostly are that request's too.
// A row's page is read from the old table entries or straight from the free
// list, so nothing waits for the new entries.  16 requests, 16 rows 5.4 us; 2048
// requests, 551,557 rows 16: waves wait two thirds of the time, for the sums, the
// search, a look-up a row, and a second round of turns for the last 5% of the rows.
constexpr int kPlanPer = 8;                         // requests of a thread
constexpr int kPlanTile = kThreads * kPlanPer;
constexpr int kPlanTurns = 4;

struct PlanArgs {
    const int32_t* kv_len;
    const int32_t* new_len;
    const int32_t* free_pages;
    const int32_t* head;
    int32_t* tables;
    int64_t* slots;
    int32_t* positions;
    int32_t* q_start;
    int32_t* kv_end;
    int32_t* head_out;
    int32_t* next_head;
    uint8_t* status;
    uint32_t* n_bad;
    int64_t n_req;
    int32_t n_free, n_tokens, max_pages, page;
    uint32_t per_page_inv;   // 2^32 / (page / 16) rounded up, 0 for 16 tokens
};

// x / page, of the tokens of a request (below 2^31 + 256).
__device__ __forceinline__ uint32_t pages_in(const PlanArgs& a, uint32_t x)
{
    return a.per_page_inv ? __umulhi(x >> 4, a.per_page_inv) : x >> 4;
}

// The last of the n ascending entries that is <= x (at[0] <= x).
__device__ __forceinline__ int last_at_most(const int32_t* at, int n, int32_t x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same for a value that all lanes of a wave have, n up to 4096.
__device__ __forceinline__ int last_at_most_wave(const int32_t* at, int n, int32_t x)
{
    const int lane = threadIdx.x & 63;
    const int step = (n + 63) >> 6;
    const int p = lane * step;
    const int lo = (__builtin_popcountll(__ballot(p < n && at[min(p, n - 1)] <= x)) - 1) * step;
    const int q = lo + lane;
    return lo + __builtin_popcountll(__ballot(lane < step && q < n && at[min(q, n - 1)] <= x)) - 1;
}

__global__ __launch_bounds__(kThreads) void page_plan_kernel(PlanArgs a)
{
    // per request of the tile: length (-1 - length if not served), first row, and the list entry of
    // its first further page
    __shared__ int32_t s_kv[kPlanTile], s_row[kPlanTile + 1], s_taken[kPlanTile];
    __shared__ uint32_t s_part[4], s_took[4], s_want[4];
    const int tid = threadIdx.x;
    const int step = (int)gridDim.x * kThreads;
    const uint32_t n_free = a.n_free, n_tokens = a.n_tokens;
    const uint32_t head0 = a.head ? min(max(*a.head, 0), a.n_free) : 0;
    uint32_t rows0 = 0;       // rows of the requests before the tile
    uint32_t need0 = head0;   // and the list entry up to which they would reach
    uint32_t took = head0;    // list entries handed out
    uint32_t want = head0;    // and asked for, up to the last request served
    for (int64_t r0 = 0; r0 < a.n_req; r0 += kPlanTile) {
        const int n = (int)min((int64_t)kPlanTile, a.n_req - r0);
        const int per = (n + kThreads - 1) / kThreads;
        int kv[kPlanPer], fresh[kPlanPer];
        uint32_t rows = 0;
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const int i = tid * per + k;
            kv[k] = fresh[k] = 0;
            if (k < per && i < n) {
                kv[k] = a.kv_len[r0 + i];
                fresh[k] = a.new_len[r0 + i];
            }
        }
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) rows = plus(rows, max(fresh[k], 0));
        uint32_t sum;
        const uint32_t first_row = plus(rows0, block_sum_before(rows, s_part, sum));
        const uint32_t rows1 = plus(rows0, sum);
        uint32_t row = first_row;
        uint32_t need = 0;
        int state[kPlanPer], pages[kPlanPer];
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const uint32_t m = max(fresh[k], 0), had = max(kv[k], 0), all = had + m;
            const uint32_t old = pages_in(a, had + a.page - 1), total = pages_in(a, min(all, kSumMost) + a.page - 1);
            row = plus(row, m);
            state[k] = kv[k] < 0 || fresh[k] < 0 || row > n_tokens ? 3 : all > kSumMost || total > (uint32_t)a.max_pages ? 2 : 0;
            pages[k] = state[k] ? 0 : (int)(total - old);
            need = plus(need, pages[k]);
        }
        uint32_t upto = plus(need0, block_sum_before(need, s_part, sum));
        const uint32_t need1 = plus(need0, sum);
        row = first_row;
        uint32_t most = took, last = want;
        int bad = 0;
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const int i = tid * per + k;
            if (k >= per || i >= n) continue;
            const uint32_t from = upto;
            upto = plus(upto, pages[k]);
            if (!state[k] && pages[k] && upto > n_free) state[k] = 1;
            const bool ok = state[k] == 0;
            if (ok && pages[k]) most = max(most, upto);
            if (ok) last = max(last, upto);
            bad += !ok;
            s_kv[i] = ok ? kv[k] : -1 - max(kv[k], 0);
            s_row[i] = (int)min(row, n_tokens);
            s_taken[i] = (int)min(from, n_free);
            if ((r0 + i) / kThreads % gridDim.x == blockIdx.x) {
                a.q_start[r0 + i] = (int)min(row, n_tokens);
                a.kv_end[r0 + i] = kv[k] + (ok ? fresh[k] : 0);
                if (a.status) a.status[r0 + i] = (uint8_t)state[k];
            }
            row = plus(row, max(fresh[k], 0));
        }
        // the last list entry handed out, and asked for, over the block
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
            most = max(most, (uint32_t)__shfl_xor((int)most, k, 64));
            last = max(last, (uint32_t)__shfl_xor((int)last, k, 64));
        }
        if ((tid & 63) == 0) s_took[tid >> 6] = most, s_want[tid >> 6] = last;
        if (tid == 0) s_row[n] = (int)min(rows1, n_tokens);
        if (blockIdx.x == 0 && a.n_bad && bad) atomicAdd(a.n_bad, (uint32_t)bad);
        __syncthreads();
        took = max(max(s_took[0], s_took[1]), max(s_took[2], s_took[3]));
        want = max(max(s_want[0], s_want[1]), max(s_want[2], s_want[3]));
        const int rows_lo = (int)min(rows0, n_tokens), rows_hi = (int)min(rows1, n_tokens);
        // this block's rows of the tile
        for (int t0 = rows_lo / step * step + (int)blockIdx.x * kThreads; t0 < rows_hi; t0 += kPlanTurns * step) {
            bool served[kPlanTurns];
            int id[kPlanTurns], off[kPlanTurns], pos[kPlanTurns];
#pragma unroll
            for (int u = 0; u < kPlanTurns; ++u) {
                const int w0 = __builtin_amdgcn_readfirstlane(t0 + u * step + (tid & ~63));   // the wave's first row
                const int t = w0 + (tid & 63);
                served[u] = false;
                id[u] = pos[u] = off[u] = 0;
                if (w0 + 63 < rows_lo || w0 >= rows_hi) continue;
                int i = last_at_most_wave(s_row, n, max(w0, rows_lo));
                if (s_row[i + 1] <= min(w0 + 63, rows_hi - 1)) i += last_at_most(s_row + i, n - i, max(t, rows_lo));
                if (t < rows_lo || t >= rows_hi) continue;
                const bool ok = s_kv[i] >= 0;
                const uint32_t had = ok ? s_kv[i] : -1 - s_kv[i];
                const uint32_t at = had + (uint32_t)(t - s_row[i]);
                const uint32_t p = pages_in(a, at), old = pages_in(a, had + a.page - 1);
                pos[u] = (int)at;
                off[u] = (int)(at - p * a.page);
                served[u] = ok;
                if (ok) id[u] = *(p < old ? a.tables + (r0 + i) * (int64_t)a.max_pages + p : a.free_pages + s_taken[i] + (p - old));
            }
#pragma unroll
            for (int u = 0; u < kPlanTurns; ++u) {
                const int t = t0 + u * step + tid;
                if (t < rows_lo || t >= rows_hi) continue;
                a.slots[t] = served[u] ? (int64_t)id[u] * a.page + off[u] : -1;
                if (a.positions) a.positions[t] = pos[u];
            }
        }
        // and its pages: list entries from need0 to took
        const int take_lo = (int)min(need0, n_free), take_hi = (int)took;
        for (int t = take_lo / step * step + (int)blockIdx.x * kThreads + tid; t < take_hi; t += step) {
            if (t < take_lo) continue;
            const int i = last_at_most(s_taken, n, t);
            const uint32_t had = s_kv[i];   // served: the entry was handed out
            a.tables[(r0 + i) * (int64_t)a.max_pages + pages_in(a, had + a.page - 1) + (t - s_taken[i])] = a.free_pages[t];
        }
        rows0 = rows1;
        need0 = need1;
        __syncthreads();
    }
    const int rest = (int)min(rows0, n_tokens);
    for (int t = rest / step * step + (int)blockIdx.x * kThreads + tid; t < a.n_tokens; t += step)
        if (t >= rest) {
            a.slots[t] = -1;
            if (a.positions) a.positions[t] = -1;
        }
    if (blockIdx.x == 0 && tid == 0) {
        a.q_start[a.n_req] = rest;
        *a.head_out = (int)want;
        if (a.next_head) *a.next_head = (int)took;
    }
}

// -------------------------------------------------------------- store, load --

// A run of rows is written by one wave for each head and each of K and V.  What
// bounds it is memory.  32,768 tokens, 8 heads of 128: 56 us (201 MB, 3.6 TB/s; 48 with
// the rows in the caches).
template <bool E4M3, bool BF16>
__global__ __launch_bounds__(kThreads, 3) void page_store_kernel(PageArgs a, Rows kr, Rows vr, int window, uint32_t* n_bad)
{
    const int64_t n_win = (a.n_tokens + window - 1) / window;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= n_win * a.heads * 2) return;
    const bool values = item & 1;
    const uint32_t hw = (uint32_t)(item >> 1);   // at most 2^31 windows x heads
    const int h = (int)(hw % (uint32_t)a.heads);
    const int64_t w0 = (int64_t)(hw / (uint32_t)a.heads) * window;
    const Rows rows = values ? vr : kr;
    const int64_t pool = a.n_pages * a.page;
    unsigned long long begins = run_begins(a, w0, window, [&](int64_t, int64_t slot) {
        if (slot >= pool && n_bad && h == 0 && !values) atomicAdd(n_bad, 1u);
    });
    while (begins) {
        const int64_t i = w0 + __builtin_ctzll(begins);
        begins &= begins - 1;
        const int64_t slot = a.slots[i];
        const int64_t page = slot / a.page;
        const int begin = (int)(slot - page * a.page);
        const int len = run_length(a, i, slot, begin);
        store_run<E4M3, BF16>(a, rows, values, i, h, page, begin, len);
    }
}

// 64 rows of the call a wave (`window`: 16 where rows are few, so that a wave's
// columns do not wait for one another), of one head and one of K and V.  The rows of one
// 16-token group that follow one another are a segment; their columns are read
// 16 at a time, keys 8 bytes a lane and row, values a channel's 16 tokens in 16
// bytes and then exchanged.  What bounds it is memory: four contexts of 32,732
// tokens, 8 heads of 128, 162 us (805 MB, 5.0 TB/s, the rate of a copy).
template <bool E4M3, bool BF16>
__global__ __launch_bounds__(kThreads) void page_load_kernel(PageArgs a, Rows kr, Rows vr, int window)
{
    __shared__ uint32_t s_seg[kThreads / 64][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c16 = lane & 15, tq = lane >> 4;
    const int64_t n_win = (a.n_tokens + window - 1) / window;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (item >= n_win * a.heads) return;
    const bool values = blockIdx.y ? true : kr.at == nullptr;
    const Rows rows = values ? vr : kr;
    const int h = (int)((uint32_t)item % (uint32_t)a.heads);
    const int64_t w0 = (int64_t)((uint32_t)item / (uint32_t)a.heads) * window;
    const uint32_t chunks = a.d / 8;
    const int64_t pool = a.n_pages * a.page;
    uint32_t* seg = s_seg[wave];

    // segments: first row, and how many
    const int n = (int)min((int64_t)window, a.n_tokens - w0);
    int64_t slot = -1;
    if (lane < n) slot = a.slots[w0 + lane];
    if (slot >= pool || slot < 0) slot = -1;
    const int64_t before = __shfl_up(slot, 1, 64);
    const bool first = lane < n && (lane == 0 || slot < 0 || (slot & 15) == 0 || before != slot - 1);
    const unsigned long long begins = __ballot(first);
    if (first) {
        const unsigned long long later = lane == 63 ? 0 : begins >> (lane + 1);
        const int len = (later ? __builtin_ctzll(later) + 1 : n - lane);
        seg[__builtin_popcountll(begins & ((1ull << lane) - 1))] = (uint32_t)lane | (uint32_t)len << 8;
    }
    wave_sync();   // the segments' lanes wrote, every lane reads
    const int columns = __builtin_popcountll(begins) * (int)chunks;
    const RowsFrom from(rows, w0, h);
    for (int base = 0; base < columns; base += 16) {
        const int col = min(base + c16, columns - 1);
        const uint32_t k = (uint32_t)col / chunks;
        const int chunk = (int)((uint32_t)col % chunks);
        const int row0 = seg[k] & 0xff, len = seg[k] >> 8;
        const int64_t sl = __shfl(slot, row0, 64);
        const int64_t at = max(sl, (int64_t)0);
        const int64_t page = (at >> 32) ? at / a.page : (uint32_t)at / (uint32_t)a.page;
        const int o = (int)(at - page * a.page);
        const float2 sc = a.scales[page * a.heads + h];
        float s = values ? sc.y : sc.x;
        const int64_t codes = (page * a.heads + h) * (int64_t)a.page * a.d;
        const int r0 = 4 * tq - (o & 15);   // this lane's first token, as a row of the segment
        uint32_t code[2][4];                // [half of the 8 channels][token]
        if (values) {
            const uint8_t* p = a.v_codes + codes + ((int64_t)(o >> 4) * a.d + 8 * chunk + tq) * 16;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 v = *(const uint4*)(p + 64 * half);
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
                exchange(w);   // channel e's tokens 4tq .. 4tq+3
#pragma unroll
                for (int j = 0; j < 4; ++j) code[half][j] = bytes_of(w, j);
            }
        } else {
            const uint8_t* p = a.k_codes + codes + (int64_t)((o >> 4) * 16 + 4 * tq) * a.d + 8 * chunk;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint2 v = *(const uint2*)(p + j * a.d);
                code[0][j] = v.x, code[1][j] = v.y;
            }
        }
        if (base + c16 >= columns) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (r0 + j < 0 || r0 + j >= len) continue;
            uint4 out = make_uint4(0, 0, 0, 0);
            if (sl >= 0) {
                float f[8];
                scaled_codes<E4M3>(code[0][j], s, f);
                scaled_codes<E4M3>(code[1][j], s, f + 4);
                out = make_uint4(f32_to_row2(f[0], f[1], BF16), f32_to_row2(f[2], f[3], BF16), f32_to_row2(f[4], f[5], BF16),
                                 f32_to_row2(f[6], f[7], BF16));
            }
            *(uint4*)(from.row(rows, row0 + r0 + j) + 16 * chunk) = out;
        }
    }
}

}  // namespace
}  // namespace fkv

using namespace fkv;

extern "C" int fkv_page_plan(int32_t page, int64_t n_req, const int32_t* kv_len, const int32_t* new_len,
                             const int32_t* free_pages, int64_t n_free, const int32_t* head, int32_t* tables,
                             int64_t max_pages, int64_t n_tokens, int64_t* slots, int32_t* positions,
                             int32_t* q_start, int32_t* kv_end, int32_t* head_out, int32_t* next_head, uint8_t* status,
                             uint32_t* n_bad, void* stream)
{
    constexpr int64_t kMost = 1 << 30;
    if (page < 16 || page > 256 || page % 16 || n_req < 0 || n_req > kMost || n_free < 0 || n_free > kMost ||
        max_pages < 1 || max_pages > (1 << 26) || n_tokens < 0 || n_tokens > kMost)
        return FKV_ERR_INVALID_ARG;
    if (!q_start || !head_out || head_out == head || (next_head && next_head == head) || !aligned(next_head, 4) || !aligned(q_start, 4) || !aligned(head_out, 4) || !aligned(head, 4) ||
        !aligned(positions, 4) || !aligned(n_bad, 4))
        return FKV_ERR_INVALID_ARG;
    if (n_req && (!kv_len || !new_len || !tables || !kv_end || kv_end == kv_len || kv_end == new_len || !aligned(kv_len, 4) || !aligned(new_len, 4) ||
                  !aligned(tables, 4) || !aligned(kv_end, 4)))
        return FKV_ERR_INVALID_ARG;
    if ((n_tokens && (!slots || !aligned(slots, 8))) || (n_free && (!free_pages || !aligned(free_pages, 4))))
        return FKV_ERR_INVALID_ARG;
    const PlanArgs a = {kv_len, new_len, free_pages, head, tables, slots, positions, q_start, kv_end,
                        head_out, next_head, status, n_bad, n_req, (int32_t)n_free, (int32_t)n_tokens, (int32_t)max_pages, page,
                        page == 16 ? 0u : (uint32_t)((((uint64_t)1 << 32) + page / 16 - 1) / (page / 16))};
    // 551,557 rows of 2048 requests: 23.2 us with 128 blocks, 17.5 with 256, 15.3 with 512, 17.6 with 1024
    const int64_t blocks = max((int64_t)1, min((int64_t)512, (n_tokens + kThreads - 1) / kThreads));
    hipLaunchKernelGGL(page_plan_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
    return launch_status();
}

extern "C" int fkv_page_store(const fkv_page_desc* desc, const fkv_row_desc* rows_k, const fkv_row_desc* rows_v,
                              const void* k_rows, const void* v_rows, int64_t n_tokens, const int64_t* slots,
                              uint8_t* k_codes, uint8_t* v_codes, float* scales, uint32_t* n_bad, void* stream)
{
    if (!page_desc_ok(desc) || !row_desc_ok(rows_k) || !row_desc_ok(rows_v) || rows_k->type != rows_v->type || n_tokens < 0 ||
        n_tokens > kMostRows)
        return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8) ||
        !aligned(n_bad, 4))
        return FKV_ERR_INVALID_ARG;
    if (n_tokens == 0) return FKV_OK;
    if (!k_rows || !v_rows || !slots || !aligned(k_rows, 16) || !aligned(v_rows, 16) || !aligned(slots, 8))
        return FKV_ERR_INVALID_ARG;
    const PageArgs a = {k_codes, v_codes, (float2*)scales, slots, n_tokens, desc->n_pages, desc->page, desc->heads, desc->d};
    // a wave looks at one row, or at a page's worth where the rows are many
    const int window = n_tokens * desc->heads <= 32768 ? 1 : min(desc->page, 64);
    const int64_t items = (n_tokens + window - 1) / window * desc->heads * 2;
    const int64_t blocks = (items + kThreads / 64 - 1) / (kThreads / 64);
    if (items > kMostBlocks) return FKV_ERR_UNSUPPORTED;
    const bool e4m3 = desc->format == FKV_PAGE_E4M3, bf16 = rows_k->type == FKV_ROW_BF16;
    auto kern = e4m3 ? bf16 ? page_store_kernel<true, true> : page_store_kernel<true, false>
                     : bf16 ? page_store_kernel<false, true> : page_store_kernel<false, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, rows_of(rows_k, k_rows),
                       rows_of(rows_v, v_rows), window, n_bad);
    return launch_status();
}

extern "C" int fkv_page_load(const fkv_page_desc* desc, const uint8_t* k_codes, const uint8_t* v_codes,
                             const float* scales, int64_t n_tokens, const int64_t* slots, const fkv_row_desc* rows_k,
                             const fkv_row_desc* rows_v, void* k_rows, void* v_rows, void* stream)
{
    if (!page_desc_ok(desc) || n_tokens < 0 || n_tokens > kMostRows || (k_rows && !row_desc_ok(rows_k)) || (v_rows && !row_desc_ok(rows_v)) ||
        (k_rows && v_rows && rows_k->type != rows_v->type))
        return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8) ||
        !aligned(k_rows, 16) || !aligned(v_rows, 16))
        return FKV_ERR_INVALID_ARG;
    if (n_tokens == 0 || (!k_rows && !v_rows)) return FKV_OK;
    if (!slots || !aligned(slots, 8)) return FKV_ERR_INVALID_ARG;
    const PageArgs a = {(uint8_t*)k_codes, (uint8_t*)v_codes, (float2*)scales, slots, n_tokens,
                        desc->n_pages, desc->page, desc->heads, desc->d};
    // with 16 and 64 rows a wave (us): 1024 tokens x 12 heads of 64 4.6 and 6.5, 2730 7.2 and 8.0, 5461 11.5 and 9.6;
    // 1024 x 8 of 128 5.5 and 8.8, 2730 8.3 and 10.5, 5461 12.5 and 14.4, 8192 17.6 and 14.1
    const int window = n_tokens * desc->heads <= 32768 ? 16 : 64;
    const int64_t items = (n_tokens + window - 1) / window * desc->heads;
    const int64_t blocks = (items + kThreads / 64 - 1) / (kThreads / 64);
    if (items > kMostBlocks) return FKV_ERR_UNSUPPORTED;
    const bool e4m3 = desc->format == FKV_PAGE_E4M3, bf16 = (k_rows ? rows_k : rows_v)->type == FKV_ROW_BF16;
    auto kern = e4m3 ? bf16 ? page_load_kernel<true, true> : page_load_kernel<true, false>
                     : bf16 ? page_load_kernel<false, true> : page_load_kernel<false, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks, k_rows && v_rows ? 2 : 1), dim3(kThreads), 0, (hipStream_t)stream, a,
                       rows_of(rows_k, k_rows), rows_of(rows_v, v_rows), window);
    return launch_status();
}
