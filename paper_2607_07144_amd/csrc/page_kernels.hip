// page_kernels.hip -- the paged 8-bit cache, for gfx950: block tables and slot
// maps from request lengths, and the writing and reading back of K/V rows.
#include "page_common.h"

namespace fkv {
namespace {

constexpr int kThreads = 256;

// --------------------------------------------------------------------- plan --

// Inclusive sum over a block's 256 threads, in thread order; `part` holds a
// word per wave.  Ends with a barrier, so `part` may be used again.
__device__ __forceinline__ int64_t block_inclusive_sum(int64_t v, int64_t* part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int64_t u = __shfl_up(v, k, 64);
        if (lane >= k) v += u;
    }
    if (lane == 63) part[wave] = v;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += part[w];
    __syncthreads();
    return v;
}

// Two prefix sums over the requests, of their rows and of the pages that they
// need, say where each row and each further page of every request goes; all
// else is a gather.  Both sums are cheap beside a second launch and a pass of
// the sums through memory, so every block forms them for itself, kPlanTile
// requests at a time in LDS, and writes its share of the rows and pages:
// kThreads consecutive ones at a time, the blocks taking turns.  The rows' and
// pages' requests are found by bisection of the sums in LDS.  A row's page is
// read from the old table entries or straight from the free list, so nothing
// waits for the new entries.
constexpr int kPlanPer = 8;                         // requests of a thread
constexpr int kPlanTile = kThreads * kPlanPer;

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
    int64_t n_req, n_free, max_pages, n_tokens;
    int32_t page;
};

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

__global__ __launch_bounds__(kThreads) void page_plan_kernel(PlanArgs a)
{
    // per request of the tile: length, first row, and the pages taken before
    // it (from the tile's first request on) with its own number of them
    __shared__ int32_t s_kv[kPlanTile], s_row[kPlanTile + 1], s_taken[kPlanTile + 1];
    __shared__ int64_t s_part[4], s_most[4], s_want[4];
    const int tid = threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * kThreads;
    const int64_t head0 = a.head ? min(max((int64_t)*a.head, (int64_t)0), a.n_free) : 0;
    int64_t rows0 = 0;       // rows of the requests before the tile
    int64_t need0 = head0;   // and the list entry up to which they would reach
    int64_t took = head0;    // list entries handed out
    int64_t want = head0;    // and asked for, up to the last request served
    for (int64_t r0 = 0; r0 < a.n_req; r0 += kPlanTile) {
        const int n = (int)min((int64_t)kPlanTile, a.n_req - r0);
        const int per = (n + kThreads - 1) / kThreads;
        int kv[kPlanPer], fresh[kPlanPer];
        int64_t rows = 0;
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const int i = tid * per + k;
            kv[k] = fresh[k] = 0;
            if (k < per && i < n) {
                kv[k] = a.kv_len[r0 + i];
                fresh[k] = a.new_len[r0 + i];
                rows += max(fresh[k], 0);
            }
        }
        int64_t row = rows0 + block_inclusive_sum(rows, s_part) - rows;
        int64_t need = 0;
        int state[kPlanPer], pages[kPlanPer];
        const int64_t first_row = row;
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const int64_t m = max(fresh[k], 0);
            const int64_t old = ((int64_t)max(kv[k], 0) + a.page - 1) / a.page;
            const int64_t all = ((int64_t)max(kv[k], 0) + m + a.page - 1) / a.page;
            state[k] = kv[k] < 0 || fresh[k] < 0 || row + m > a.n_tokens ? 3 : all > a.max_pages || kv[k] + m > 0x7fffffff ? 2 : 0;
            pages[k] = state[k] ? 0 : (int)(all - old);
            need += pages[k];
            row += m;
        }
        int64_t upto = need0 + block_inclusive_sum(need, s_part);
        if (tid == kThreads - 1) {
            s_most[0] = row;    // the tile's totals, for the next
            s_most[1] = upto;
        }
        upto -= need;
        row = first_row;
        int64_t most = took, last = want;
        int bad = 0;
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const int i = tid * per + k;
            if (k >= per || i >= n) continue;
            const int64_t from = upto;
            upto += pages[k];
            if (!state[k] && pages[k] && upto > a.n_free) state[k] = 1;
            const bool ok = state[k] == 0;
            if (ok && pages[k]) most = max(most, upto);
            if (ok) last = max(last, upto);
            bad += !ok;
            s_kv[i] = ok ? kv[k] : -1 - max(kv[k], 0);
            s_row[i] = (int)min(row, a.n_tokens);
            s_taken[i] = (int)min(from, a.n_free);   // of those served: the list entry of the first page
            if ((r0 + i) / kThreads % gridDim.x == blockIdx.x) {
                a.q_start[r0 + i] = (int)min(row, a.n_tokens);
                a.kv_end[r0 + i] = kv[k] + (ok ? fresh[k] : 0);
                if (a.status) a.status[r0 + i] = (uint8_t)state[k];
            }
            row += max(fresh[k], 0);
        }
        // the last list entry handed out, and asked for, over the block
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
            most = max(most, (int64_t)__shfl_xor(most, k, 64));
            last = max(last, (int64_t)__shfl_xor(last, k, 64));
        }
        if ((tid & 63) == 0) s_part[tid >> 6] = most, s_want[tid >> 6] = last;
        if (blockIdx.x == 0 && a.n_bad && bad) atomicAdd(a.n_bad, (uint32_t)bad);
        __syncthreads();
        const int64_t rows1 = s_most[0], need1 = s_most[1];
        took = max(max(s_part[0], s_part[1]), max(s_part[2], s_part[3]));
        want = max(max(s_want[0], s_want[1]), max(s_want[2], s_want[3]));
        const int rows_lo = (int)min(rows0, a.n_tokens), rows_hi = (int)min(rows1, a.n_tokens);
        // this block's rows of the tile
        for (int64_t t = rows_lo / step * step + (int64_t)blockIdx.x * kThreads + tid; t < rows_hi; t += step) {
            if (t < rows_lo) continue;
            const int i = last_at_most(s_row, n, (int)t);
            const int off = (int)t - s_row[i];
            const bool ok = s_kv[i] >= 0;
            const int had = ok ? s_kv[i] : -1 - s_kv[i];
            const int pos = (int)((int64_t)had + off);
            int64_t slot = -1;
            if (ok) {
                const int p = pos / a.page, old = (had + a.page - 1) / a.page;
                const int id = p < old ? a.tables[(r0 + i) * a.max_pages + p] : a.free_pages[s_taken[i] + p - old];
                slot = (int64_t)id * a.page + pos % a.page;
            }
            a.slots[t] = slot;
            if (a.positions) a.positions[t] = pos;
        }
        // and its pages: list entries [need0, took)
        const int take_lo = (int)min(need0, a.n_free), take_hi = (int)took;
        for (int64_t t = take_lo / step * step + (int64_t)blockIdx.x * kThreads + tid; t < take_hi; t += step) {
            if (t < take_lo) continue;
            const int i = last_at_most(s_taken, n, (int)t);
            const int had = s_kv[i];   // served: the entry was handed out
            a.tables[(r0 + i) * a.max_pages + (had + a.page - 1) / a.page + (t - s_taken[i])] = a.free_pages[t];
        }
        rows0 = rows1;
        need0 = need1;
        __syncthreads();
    }
    for (int64_t t = rows0 / step * step + (int64_t)blockIdx.x * kThreads + tid; t < a.n_tokens; t += step)
        if (t >= rows0) {
            a.slots[t] = -1;
            if (a.positions) a.positions[t] = -1;
        }
    if (blockIdx.x == 0 && tid == 0) {
        a.q_start[a.n_req] = (int)min(rows0, a.n_tokens);
        *a.head_out = (int)min(want, (int64_t)0x7fffffff);
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
    __device__ __forceinline__ uint8_t* row(int64_t i, int h) const
    {
        const int64_t g = group > i ? 0 : i / group;
        return at + 2 * (g * stride_group + (i - g * group) * stride_token + h * stride_head);
    }
};

// A run of rows whose slots follow one another within a page is written by one
// wave for each head and each of K and V.  A lane holds a quad -- the same 8
// channels of 4 tokens whose offsets are 4q .. 4q+3 -- so that four value codes
// of a channel, which lie side by side, go out as one word; `page` * d up to 8192
// elements stay in registers between the largest element and the codes, larger
// pages are read a second time (from the caches).
constexpr int kQuads = 4;             // quads of a lane held in registers
constexpr int kHeld = kQuads * 64;    // quads of a wave

struct Quad {
    uint4 row[4];
};

template <bool E4M3>
__global__ __launch_bounds__(kThreads) void page_store_kernel(PageArgs a, Rows kr, Rows vr, int bf16, int window,
                                                              uint32_t* n_bad)
{
    const int lane = threadIdx.x & 63;
    const int64_t n_win = (a.n_tokens + window - 1) / window;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (item >= n_win * a.heads * 2) return;
    const bool values = item & 1;
    const int h = (int)((item >> 1) % a.heads);
    const int64_t w0 = (item >> 1) / a.heads * window;
    const int64_t w1 = min(w0 + window, a.n_tokens);
    const Rows rows = values ? vr : kr;
    const int chunks = a.d / 8;
    const int64_t pool = a.n_pages * a.page;
    const float largest = E4M3 ? kLargestE4m3 : kLargestInt8;
    for (int64_t i = w0; i < w1; ++i) {
        const int64_t slot = a.slots[i];
        if (slot < 0) continue;
        if (slot >= pool) {
            if (n_bad && h == 0 && !values && lane == 0) atomicAdd(n_bad, 1u);
            continue;
        }
        const int64_t page = slot / a.page;
        const int begin = (int)(slot - page * a.page);
        // its run starts at the page's first token or where the row before it does not lead up to it
        if (begin && i && a.slots[i - 1] == slot - 1) continue;
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
        const int q0 = begin >> 2, n_quads = ((end + 3) >> 2) - q0;   // quads that hold some of the run
        const int tasks = n_quads * chunks;
        auto load = [&](int task, Quad& x) {
            const int q = q0 + task / chunks, c = task % chunks;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int o = 4 * q + j;
                x.row[j] = make_uint4(0, 0, 0, 0);
                if (task < tasks && o >= begin && o < end)
                    x.row[j] = *(const uint4*)(rows.row(i + (o - begin), h) + 16 * c);
            }
        };
        // the run's largest finite element
        Quad held[kQuads];
        float most = 0.0f;
        for (int base = 0; base < tasks; base += kHeld) {
#pragma unroll
            for (int u = 0; u < kQuads; ++u) load(base + u * 64 + lane, held[u]);
#pragma unroll
            for (int u = 0; u < kQuads; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t word = e < 2 ? held[u].row[j].x : e < 4 ? held[u].row[j].y : e < 6 ? held[u].row[j].z : held[u].row[j].w;
                        const float f = fabsf(row_to_f32(word, e & 1, bf16));
                        most = fmaxf(most, f < __builtin_inff() ? f : 0.0f);
                    }
        }
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) most = fmaxf(most, __shfl_xor(most, k, 64));
        float* sp = (float*)&a.scales[page * a.heads + h] + (values ? 1 : 0);
        float s = most < 0x1p-90f ? 0.0f : most * (1.0f / largest);
        uint8_t* codes = (values ? a.v_codes : a.k_codes) + (page * a.heads + h) * (int64_t)a.page * a.d;
        if (begin) {
            const float was = *sp;
            s = fmaxf(s, was);
            if (s > was) {
                // the tokens before the run at the new scale; of a quad that the run begins in, only their bytes
                const float grow = was / s;
                const int words = values ? q0 * a.d + (begin & 3 ? a.d : 0) : begin * (a.d / 4);
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
        if (lane == 0) *sp = s;
        const float inv = s > 0.0f ? 1.0f / s : 0.0f;
        for (int base = 0; base < tasks; base += kHeld) {
            if (tasks > kHeld) {
#pragma unroll
                for (int u = 0; u < kQuads; ++u) load(base + u * 64 + lane, held[u]);
            }
#pragma unroll
            for (int u = 0; u < kQuads; ++u) {
                const int task = base + u * 64 + lane;
                if (task >= tasks) continue;
                const int q = q0 + task / chunks, c = task % chunks;
                uint32_t code[4][2];   // [token][half of the 8 channels]
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t lo = half ? held[u].row[j].z : held[u].row[j].x;
                        const uint32_t hi = half ? held[u].row[j].w : held[u].row[j].y;
                        float f[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = row_to_f32(e < 2 ? lo : hi, e & 1, bf16);
                            f[e] = fabsf(x) < __builtin_inff() ? x * inv : x != x ? 0.0f : copysignf(largest, x);
                        }
                        code[j][half] = f32_to_codes<E4M3>(f);
                    }
                const bool whole = 4 * q >= begin && 4 * q + 4 <= end;
                if (!values) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int o = 4 * q + j;
                        if (o >= begin && o < end)
                            *(uint2*)(codes + o * a.d + 8 * c) = make_uint2(code[j][0], code[j][1]);
                    }
                } else {
                    uint8_t* at = codes + ((int64_t)(q >> 2) * a.d + 8 * c) * 16 + 4 * (q & 3);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        uint32_t word = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) word |= ((code[j][e >> 2] >> (8 * (e & 3))) & 0xff) << (8 * j);
                        if (whole)
                            *(uint32_t*)(at + 16 * e) = word;
                        else
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (4 * q + j >= begin && 4 * q + j < end) at[16 * e + j] = (uint8_t)(word >> (8 * j));
                    }
                }
            }
        }
    }
}

// Four consecutive rows of the call by 8 channels a lane: where their slots are
// a quad of a page the value codes come as words, else byte by byte.
template <bool E4M3>
__global__ __launch_bounds__(kThreads) void page_load_kernel(PageArgs a, Rows kr, Rows vr, int bf16)
{
    const int chunks = a.d / 8;
    const int64_t n_quads = (a.n_tokens + 3) / 4;
    const int64_t task = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (task >= n_quads * chunks * a.heads) return;
    const bool values = blockIdx.y ? true : kr.at == nullptr;
    const Rows rows = values ? vr : kr;
    const int c = (int)(task % chunks);
    const int h = (int)(task / chunks % a.heads);
    const int64_t i0 = task / chunks / a.heads * 4;
    const int64_t pool = a.n_pages * a.page;
    uint32_t code[4][2];
    float scale[4];
    int64_t slot[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        slot[j] = i0 + j < a.n_tokens ? a.slots[i0 + j] : -1;
        if (slot[j] >= pool) slot[j] = -1;
    }
    const bool quad = slot[0] >= 0 && slot[0] % 4 == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 && slot[3] == slot[0] + 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        code[j][0] = code[j][1] = 0;
        scale[j] = 0.0f;
        if (slot[j] < 0) continue;
        const int64_t page = slot[j] / a.page;
        const int o = (int)(slot[j] - page * a.page);
        const float2 sc = a.scales[page * a.heads + h];
        scale[j] = values ? sc.y : sc.x;
        const int64_t base = (page * a.heads + h) * (int64_t)a.page * a.d;
        if (!values) {
            const uint2 w = *(const uint2*)(a.k_codes + base + o * a.d + 8 * c);
            code[j][0] = w.x, code[j][1] = w.y;
        } else if (!quad) {
            const uint8_t* at = a.v_codes + base + ((int64_t)(o >> 4) * a.d + 8 * c) * 16 + (o & 15);
#pragma unroll
            for (int e = 0; e < 8; ++e) code[j][e >> 2] |= (uint32_t)at[16 * e] << (8 * (e & 3));
        }
    }
    if (values && quad) {
        const int64_t page = slot[0] / a.page;
        const int o = (int)(slot[0] - page * a.page);
        const uint8_t* at = a.v_codes + (page * a.heads + h) * (int64_t)a.page * a.d + ((int64_t)(o >> 4) * a.d + 8 * c) * 16 + (o & 15);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t w = *(const uint32_t*)(at + 16 * e);
#pragma unroll
            for (int j = 0; j < 4; ++j) code[j][e >> 2] |= ((w >> (8 * j)) & 0xff) << (8 * (e & 3));
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (i0 + j >= a.n_tokens) break;
        float f[4], g[4];
        codes_to_f32<E4M3>(code[j][0], f);
        codes_to_f32<E4M3>(code[j][1], g);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] *= scale[j], g[e] *= scale[j];
        *(uint4*)(rows.row(i0 + j, h) + 16 * c) =
            make_uint4(f32_to_row2(f[0], f[1], bf16), f32_to_row2(f[2], f[3], bf16), f32_to_row2(g[0], g[1], bf16),
                       f32_to_row2(g[2], g[3], bf16));
    }
}

Rows rows_of(const fkv_row_desc* r, const void* at)
{
    if (!at) return Rows{nullptr, 1, 0, 0, 0};
    return Rows{(uint8_t*)at, r->group, r->stride_group, r->stride_token, r->stride_head};
}

constexpr int64_t kMostBlocks = 0x7fffff00;

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
                        head_out, next_head, status, n_bad, n_req, n_free, max_pages, n_tokens, page};
    const int64_t blocks = max((int64_t)1, min((int64_t)256, (n_tokens + kThreads - 1) / kThreads));
    hipLaunchKernelGGL(page_plan_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
    return launch_status();
}

extern "C" int fkv_page_store(const fkv_page_desc* desc, const fkv_row_desc* rows_k, const fkv_row_desc* rows_v,
                              const void* k_rows, const void* v_rows, int64_t n_tokens, const int64_t* slots,
                              uint8_t* k_codes, uint8_t* v_codes, float* scales, uint32_t* n_bad, void* stream)
{
    if (!page_desc_ok(desc) || !row_desc_ok(rows_k) || !row_desc_ok(rows_v) || rows_k->type != rows_v->type || n_tokens < 0)
        return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8) ||
        !aligned(n_bad, 4))
        return FKV_ERR_INVALID_ARG;
    if (n_tokens == 0) return FKV_OK;
    if (!k_rows || !v_rows || !slots || !aligned(k_rows, 16) || !aligned(v_rows, 16) || !aligned(slots, 8))
        return FKV_ERR_INVALID_ARG;
    const PageArgs a = {k_codes, v_codes, (float2*)scales, slots, n_tokens, desc->n_pages, desc->page, desc->heads, desc->d};
    // a wave looks at one row, or at 16 where the rows are many
    const int window = n_tokens <= 1024 ? 1 : 16;
    const int64_t items = (n_tokens + window - 1) / window * desc->heads * 2;
    const int64_t blocks = (items + kThreads / 64 - 1) / (kThreads / 64);
    if (blocks > kMostBlocks) return FKV_ERR_UNSUPPORTED;
    auto kern = desc->format == FKV_PAGE_E4M3 ? page_store_kernel<true> : page_store_kernel<false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, rows_of(rows_k, k_rows),
                       rows_of(rows_v, v_rows), (int)rows_k->type, window, n_bad);
    return launch_status();
}

extern "C" int fkv_page_load(const fkv_page_desc* desc, const uint8_t* k_codes, const uint8_t* v_codes,
                             const float* scales, int64_t n_tokens, const int64_t* slots, const fkv_row_desc* rows_k,
                             const fkv_row_desc* rows_v, void* k_rows, void* v_rows, void* stream)
{
    if (!page_desc_ok(desc) || n_tokens < 0 || (k_rows && !row_desc_ok(rows_k)) || (v_rows && !row_desc_ok(rows_v)) ||
        (k_rows && v_rows && rows_k->type != rows_v->type))
        return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8) ||
        !aligned(k_rows, 16) || !aligned(v_rows, 16))
        return FKV_ERR_INVALID_ARG;
    if (n_tokens == 0 || (!k_rows && !v_rows)) return FKV_OK;
    if (!slots || !aligned(slots, 8)) return FKV_ERR_INVALID_ARG;
    const PageArgs a = {(uint8_t*)k_codes, (uint8_t*)v_codes, (float2*)scales, slots, n_tokens,
                        desc->n_pages, desc->page, desc->heads, desc->d};
    const int64_t tasks = (n_tokens + 3) / 4 * (desc->d / 8) * desc->heads;
    const int64_t blocks = (tasks + kThreads - 1) / kThreads;
    if (blocks > kMostBlocks) return FKV_ERR_UNSUPPORTED;
    const int type = k_rows ? rows_k->type : rows_v->type;
    auto kern = desc->format == FKV_PAGE_E4M3 ? page_load_kernel<true> : page_load_kernel<false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks, k_rows && v_rows ? 2 : 1), dim3(kThreads), 0, (hipStream_t)stream, a,
                       rows_of(rows_k, k_rows), rows_of(rows_v, v_rows), type);
    return launch_status();
}
