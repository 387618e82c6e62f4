// page_kernels.hip -- the paged 8-bit cache, for gfx950: block tables and slot
// maps from request lengths, and the writing and reading back of K/V rows.
#include "page_common.h"

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

struct PageArgs {
    uint8_t* k_codes;
    uint8_t* v_codes;
    float2* scales;
    const int64_t* slots;
    int64_t n_tokens, n_pages;
    int32_t page, heads, d;
};

struct Rows {
    uint8_t* at;
    int64_t group, stride_group, stride_token, stride_head;
};

// Rows near a first one, with one division for all that lie in its group.
struct RowsFrom {
    uint8_t* at;       // of the first row
    int64_t left;      // rows from it to the end of its group
    __device__ __forceinline__ RowsFrom(const Rows& r, int64_t i, int h)
    {
        const int64_t g = r.group > i ? 0 : (i >> 32 | r.group >> 32) ? i / r.group : (uint32_t)i / (uint32_t)r.group;
        left = r.group - (i - g * r.group);
        at = r.at + 2 * (g * r.stride_group + (i - g * r.group) * r.stride_token + h * r.stride_head);
    }
    __device__ __forceinline__ uint8_t* row(const Rows& r, int k) const
    {
        uint8_t* p = at + 2 * k * r.stride_token;
        if (k >= left) {   // k - left rows into a later group
            const int64_t g = 1 + (k - left) / r.group;
            p += 2 * g * (r.stride_group - r.group * r.stride_token);
        }
        return p;
    }
};

// Both kernels give a lane a column -- 8 channels of a 16-token group -- and
// four of its tokens: lane 16q + c holds tokens 4q .. 4q+3 of column c, as rows
// of 16 bytes.  In the values' layout a channel's 16 tokens lie side by side;
// this is the 4 x 4 exchange between the two, of 32-bit words over the four
// 16-lane rows of a wave.  Word e of row q goes to word q of row e.
__device__ __forceinline__ void exchange(uint32_t (&w)[4])
{
    auto swap32 = [](uint32_t& a, uint32_t& b) {
        const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        a = r[0], b = r[1];
    };
    auto swap16 = [](uint32_t& a, uint32_t& b) {
        const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        a = r[0], b = r[1];
    };
    swap32(w[0], w[2]);
    swap32(w[1], w[3]);
    swap16(w[0], w[1]);
    swap16(w[2], w[3]);
}

// Byte e of four words as one word.
__device__ __forceinline__ uint32_t bytes_of(const uint32_t (&w)[4], int e)
{
    const uint32_t sel = 0x0c0c0000u | (uint32_t)(e << 8) | (uint32_t)(4 + e);   // of the second and the first argument
    const uint32_t lo = __builtin_amdgcn_perm(w[0], w[1], sel);
    const uint32_t hi = __builtin_amdgcn_perm(w[2], w[3], sel);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// A run of rows whose slots follow one another within a page is written by one
// wave for each head and each of K and V, up to 64 columns of it (a page of 64
// tokens x 128 channels) held in registers between the largest element and the
// codes; larger pages are read a second time (from the caches).  What bounds it
// is memory: rows are read 16 bytes a lane, codes written 8 (keys) and 16
// (values) bytes a lane.  The largest element is found on the rows' bits, two at
// a time: without the sign they are in the order of the numbers, and what is
// not finite comes last; only a run that has such elements looks at each.  32,768
// tokens, 8 heads of 128: 56 us (201 MB, 3.6 TB/s; 48 with the rows in the caches).
constexpr int kPasses = 4;   // of 16 columns

template <bool E4M3, bool BF16>
__global__ __launch_bounds__(kThreads, 3) void page_store_kernel(PageArgs a, Rows kr, Rows vr, int window, uint32_t* n_bad)
{
    typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
    constexpr uint32_t kInf = BF16 ? 0x7f80 : 0x7c00;
    constexpr float kLargest = E4M3 ? kLargestE4m3 : kLargestInt8;
    const int lane = threadIdx.x & 63, c16 = lane & 15, tq = lane >> 4;
    const int64_t n_win = (a.n_tokens + window - 1) / window;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= n_win * a.heads * 2) return;
    const bool values = item & 1;
    const uint32_t hw = (uint32_t)(item >> 1);   // at most 2^31 windows x heads
    const int h = (int)(hw % (uint32_t)a.heads);
    const int64_t w0 = (int64_t)(hw / (uint32_t)a.heads) * window;
    const Rows rows = values ? vr : kr;
    const uint32_t chunks = a.d / 8;
    const int64_t pool = a.n_pages * a.page;

    // the rows of the window that begin a run: at a page's first token, or where the row before does not lead up to them
    unsigned long long begins;
    {
        const int64_t i = w0 + lane;
        bool first = false;
        if (lane < window && i < a.n_tokens) {
            const int64_t slot = a.slots[i], before = i ? a.slots[i - 1] : -2;
            first = slot >= 0 && slot < pool && ((uint32_t)(slot % a.page) == 0 || before != slot - 1);
            if (slot >= pool && n_bad && h == 0 && !values) atomicAdd(n_bad, 1u);
        }
        begins = __ballot(first);
    }
    while (begins) {
        const int64_t i = w0 + __builtin_ctzll(begins);
        begins &= begins - 1;
        const int64_t slot = a.slots[i];
        const int64_t page = slot / a.page;
        const int begin = (int)(slot - page * a.page);
        int len = 1;
        {
            const int most = (int)min((int64_t)(a.page - begin), a.n_tokens - i);
            for (int base = 1; base < most; base += 64) {
                const bool follows = base + lane < most && a.slots[i + base + lane] == slot + base + lane;
                const unsigned long long m = __ballot(!follows);
                const int run = m ? __builtin_ctzll(m) : 64;
                len = base + run;
                if (run < 64) break;
            }
        }
        const int end = begin + len;
        const int g0 = begin >> 4;
        const int columns = (((end + 15) >> 4) - g0) * chunks;
        const RowsFrom from(rows, i, h);
        // this lane's tokens of a column: offsets first .. first+3 in the page
        auto place = [&](int col, int& grp, int& chunk) {
            grp = g0 + (int)((uint32_t)col / chunks);
            chunk = (int)((uint32_t)col % chunks);
        };
        uint4 held[kPasses][4];
        auto load = [&](int base) {
#pragma unroll
            for (int u = 0; u < kPasses; ++u) {
                const int col = base + u * 16 + c16;
                int grp, chunk;
                place(col, grp, chunk);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int o = grp * 16 + tq * 4 + j;
                    held[u][j] = make_uint4(0, 0, 0, 0);
                    if (col < columns && o >= begin && o < end) held[u][j] = *(const uint4*)(from.row(rows, o - begin) + 16 * chunk);
                }
            }
        };
        // the largest of the rows' bits, and of those of finite elements
        ushort2_t top = {0, 0};
        for (int base = 0; base < columns; base += 16 * kPasses) {
            load(base);
#pragma unroll
            for (int u = 0; u < kPasses; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w[4] = {held[u][j].x, held[u][j].y, held[u][j].z, held[u][j].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort2_t, w[e] & 0x7fff7fffu));
                }
        }
        uint32_t most = max((uint32_t)top[0], (uint32_t)top[1]);
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, k, 64));
        const bool special = most >= kInf;
        if (special) {
            most = 0;
            for (int base = 0; base < columns; base += 16 * kPasses) {
                load(base);
#pragma unroll
                for (int u = 0; u < kPasses; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t w[4] = {held[u][j].x, held[u][j].y, held[u][j].z, held[u][j].w};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t b = (w[e >> 1] >> (16 * (e & 1))) & 0x7fff;
                            most = max(most, b < kInf ? b : 0u);
                        }
                    }
            }
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, k, 64));
        }
        const float largest = row_to_f32(most, 0, BF16);
        float* sp = (float*)&a.scales[page * a.heads + h] + (values ? 1 : 0);
        float s = largest < 0x1p-90f ? 0.0f : largest * (1.0f / kLargest);
        uint8_t* codes = (values ? a.v_codes : a.k_codes) + (page * a.heads + h) * (int64_t)a.page * a.d;
        if (begin) {
            const float was = *sp;
            s = fmaxf(s, was);
            if (s > was) {
                // the tokens before the run at the new scale; of a quad that the run begins in, only their bytes
                const float grow = was / s;
                const int quads = begin >> 2;
                const int words = values ? (quads + (begin & 3 ? 1 : 0)) * a.d : begin * (a.d / 4);
                for (int t = lane; t < words; t += 64) {
                    uint32_t* at;
                    int keep = 4;
                    if (values) {
                        const int q = t / a.d, e = t % a.d;   // quad and channel
                        at = (uint32_t*)(codes + ((int64_t)(q >> 2) * a.d + e) * 16) + (q & 3);
                        keep = min(4, begin - 4 * q);
                    } else {
                        at = (uint32_t*)codes + t;
                    }
                    float f[4];
                    codes_to_f32<E4M3>(*at, f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] *= grow;
                    const uint32_t c = f32_to_codes<E4M3>(f);
                    if (keep == 4)
                        *at = c;
                    else
                        for (int e = 0; e < keep; ++e) ((uint8_t*)at)[e] = (uint8_t)(c >> (8 * e));
                }
            }
        }
        wave_sync();   // every lane has read the scale, and words of which others write bytes
        if (lane == 0) *sp = s;
        const float inv = s > 0.0f ? 1.0f / s : 0.0f;
        for (int base = 0; base < columns; base += 16 * kPasses) {
            if (columns > 16 * kPasses || special) load(base);
#pragma unroll
            for (int u = 0; u < kPasses; ++u) {
                if (base + u * 16 >= columns) break;
                const int col = base + u * 16 + c16;
                int grp, chunk;
                place(col, grp, chunk);
                const int o0 = grp * 16 + tq * 4;
                uint32_t code[2][4];   // [half of the 8 channels][token]
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t lo = half ? held[u][j].z : held[u][j].x;
                        const uint32_t hi = half ? held[u][j].w : held[u][j].y;
                        float f[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) f[e] = row_to_f32(e < 2 ? lo : hi, e & 1, BF16) * inv;
                        if (special) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float x = row_to_f32(e < 2 ? lo : hi, e & 1, BF16);
                                f[e] = fabsf(x) < __builtin_inff() ? f[e] : x != x ? 0.0f : copysignf(kLargest, x);
                            }
                        }
                        code[half][j] = near_codes<E4M3>(f);
                    }
                if (!values) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (col < columns && o0 + j >= begin && o0 + j < end)
                            *(uint2*)(codes + (o0 + j) * a.d + 8 * chunk) = make_uint2(code[0][j], code[1][j]);
                    continue;
                }
                const bool whole = grp * 16 >= begin && grp * 16 + 16 <= end;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t w[4];   // channel e of the half: its four tokens here, then channel tq's sixteen
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = bytes_of(code[half], e);
                    exchange(w);
                    if (col >= columns) continue;
                    uint8_t* at = codes + ((int64_t)grp * a.d + 8 * chunk + 4 * half + tq) * 16;
                    if (whole) {
                        *(uint4*)at = make_uint4(w[0], w[1], w[2], w[3]);
                        continue;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int b = grp * 16 + 4 * q;
                        if (b >= begin && b + 4 <= end)
                            *(uint32_t*)(at + 4 * q) = w[q];
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (b + e >= begin && b + e < end) at[4 * q + e] = (uint8_t)(w[q] >> (8 * e));
                    }
                }
            }
        }
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

Rows rows_of(const fkv_row_desc* r, const void* at)
{
    if (!at) return Rows{nullptr, 1, 0, 0, 0};
    return Rows{(uint8_t*)at, r->group, r->stride_group, r->stride_token, r->stride_head};
}

constexpr int64_t kMostBlocks = 0x7fffff00;
constexpr int64_t kMostRows = (int64_t)1 << 40;   // beyond any memory; times the heads it is a number of 64 bits

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
