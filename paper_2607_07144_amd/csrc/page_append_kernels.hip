// page_append_kernels.hip -- rows on their way into the paged cache, for gfx950:
// query and key rows rotated by their positions, K/V rows written into pages, and
// the boxes of the pages' keys kept up to date, in one launch.
//
// A rotation turns pairs of channels (a, b) of a row by the angle of its position
// and pair:  a' = a c - b s,  b' = b c + a s,  with (c, s) from a table, each
// product and sum rounded to fp32.  Keys are never rounded to their type in
// between: their scale and codes come from the fp32 values.
//
// A page's box is the smallest and the largest code of each key channel over its
// tokens.  Rounding to codes is monotone, so a channel's ends are those of the new
// rows, rounded, and of the codes before them.  Those are read each time, and the box
// that was there is not: tokens that are written over, as of drafts that were refused,
// are in it.
#include "page_rows_device.h"

#include <algorithm>

namespace fkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr float kInf = __builtin_inff();
constexpr int kBoxRow = 64 + 8;   // an element's row of 64 lanes in LDS (8 more: the elements of a chunk lie in banks of their own)

struct AppendArgs {
    Rows q, q_out, k, v;
    const int32_t* positions;
    const float4* table;   // two pairs' (c, s) at a time
    uint8_t* boxes;
    uint32_t* n_bad;
    int64_t n_pos;
    int64_t store_items;   // windows x heads x (K, V): a wave each
    int64_t q_lanes;       // tokens x groups of query heads x units: a lane each
    int32_t window, q_heads, q_groups;
    int32_t rot;
    bool pairs;
};

// Channels are taken in units of 16, two chunks of 8 that hold eight pairs: of
// rotated channels c and c + rot/2 the unit's chunks lie rot/2 apart, else they are
// neighbours.  The table's entries of unit u are 8u .. 8u+7 either way.
struct Unit {
    int c0, c1;     // chunks
    bool turned;
};

__device__ __forceinline__ Unit unit_of(const AppendArgs& p, int u)
{
    const int half = p.rot >> 4;
    const bool apart = !p.pairs && u < half;
    return Unit{apart ? u : 2 * u, apart ? u + half : 2 * u + 1, u < half};
}

__device__ __forceinline__ int table_row(const AppendArgs& p, int64_t i)
{
    return (int)min(max((int64_t)p.positions[i], (int64_t)0), p.n_pos - 1);
}

// 16 elements of a unit in fp32, turned by the table's eight entries.
template <bool BF16>
__device__ __forceinline__ void turn(uint4 lo, uint4 hi, const float4 (&cs)[4], bool turned, bool pairs, float (&f)[16])
{
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = row_to_f32(w[e >> 1], e & 1, BF16);
    if (!turned) return;
    if (pairs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = e & 1 ? cs[e >> 1].z : cs[e >> 1].x, s = e & 1 ? cs[e >> 1].w : cs[e >> 1].y;
            const float a = f[2 * e], b = f[2 * e + 1];
            f[2 * e] = a * c - b * s;
            f[2 * e + 1] = b * c + a * s;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = e & 1 ? cs[e >> 1].z : cs[e >> 1].x, s = e & 1 ? cs[e >> 1].w : cs[e >> 1].y;
            const float a = f[e], b = f[8 + e];
            f[e] = a * c - b * s;
            f[8 + e] = b * c + a * s;
        }
    }
}

// What a lane has of a run's key rows: one unit of every `slots`-th token from `first`.
struct KeyLane {
    Unit unit;
    int u, slots, slot;
    bool used;
    __device__ __forceinline__ KeyLane(const AppendArgs& p, int units)
    {
        const int lane = threadIdx.x & 63;
        slots = 64 / units;
        slot = lane / units;
        u = lane - slot * units;
        used = slot < slots;
        unit = unit_of(p, u);
    }
};

// The codes of a page's keys before `begin`, as the lanes have the new rows: a lane its unit
// of every `slots`-th token, kTurns tokens in flight, for a box the first ones read before
// the new scale is known.  (Reading them for each box, not only where the scale grows: a token of each
// of 64 requests with half full pages of 64 x 128, 8 heads, 8.0 -> 9.4 us, of 4096 requests
// 185 -> 196; 12 ragged prompts 45.5 -> 47.1.)
template <bool E4M3>
struct OldKeys {
    static constexpr int kTurns = 4;
    uint8_t* codes;
    int d, begin;
    bool ahead;
    uint2 lo[kTurns], hi[kTurns];
    __device__ __forceinline__ OldKeys(uint8_t* codes_, int d_, int begin_, bool ahead_, const KeyLane& mine)
        : codes(codes_), d(d_), begin(begin_), ahead(ahead_)
    {
        if (begin && ahead) fetch(0, mine);
    }
    __device__ __forceinline__ void fetch(int k0, const KeyLane& mine)
    {
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const uint8_t* at = codes + min(k0 + t * mine.slots + mine.slot, begin - 1) * d;
            lo[t] = *(const uint2*)(at + 8 * mine.unit.c0);
            hi[t] = *(const uint2*)(at + 8 * mine.unit.c1);
        }
    }
    // all of them times `grow`, back to where they were; `each` is told the codes as they are then, the last token's where a
    // lane has none left
    template <typename F>
    __device__ __forceinline__ void rescale(float grow, const KeyLane& mine, F each)
    {
        for (int k0 = 0; k0 < begin; k0 += kTurns * mine.slots) {
            if (k0 || !ahead) fetch(k0, mine);
            uint32_t w[kTurns][4];
#pragma unroll
            for (int t = 0; t < kTurns; ++t) w[t][0] = lo[t].x, w[t][1] = lo[t].y, w[t][2] = hi[t].x, w[t][3] = hi[t].y;
            if (grow != 1.0f) {
#pragma unroll
                for (int t = 0; t < kTurns; ++t) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[t][q] = grown<E4M3>(w[t][q], grow);
                    const int k = k0 + t * mine.slots + mine.slot;
                    if (!mine.used || k >= begin) continue;
                    uint8_t* to = codes + k * d;
                    *(uint2*)(to + 8 * mine.unit.c0) = make_uint2(w[t][0], w[t][1]);
                    *(uint2*)(to + 8 * mine.unit.c1) = make_uint2(w[t][2], w[t][3]);
                }
            }
            each(w);
        }
    }
};

// A wave writes a run of one head's keys, as store_run does, turned on the way.  It takes
// 64 / units tokens T times over in a pass (16 tokens of 128 channels), which is held in
// registers between the channels' smallest and largest values -- and with them the largest
// of all -- and the codes; of a run of more the rows are read and turned a second time,
// from the caches.
template <bool E4M3, bool BF16>
__device__ __forceinline__ void append_keys(const PageArgs& a, const AppendArgs& p, float* s_box, int64_t i, int h, int64_t page,
                                            int begin, int len)
{
    constexpr float kLargest = E4M3 ? kLargestE4m3 : kLargestInt8;
    constexpr int T = 2;
    const int lane = threadIdx.x & 63;
    const int d = a.d, units = d >> 4;
    float* sp = (float*)&a.scales[page * a.heads + h];
    uint8_t* codes = a.k_codes + (page * a.heads + h) * (int64_t)a.page * d;
    const float was = begin ? *sp : 0.0f;
    const KeyLane mine(p, units);
    OldKeys<E4M3> before(codes, d, begin, p.boxes != nullptr, mine);
    const RowsFrom from(p.k, i, h);
    const int per_pass = mine.slots * T;
    const int n_pass = (len + per_pass - 1) / per_pass;
    auto token = [&](int pass, int j) { return pass * per_pass + j * mine.slots + mine.slot; };   // of the run
    auto there = [&](int k) { return mine.used && k < len; };
    float held[T][16];
    auto load = [&](int pass) {
        uint4 lo[T], hi[T];
        int row[T];
#pragma unroll
        for (int j = 0; j < T; ++j) {
            lo[j] = hi[j] = make_uint4(0, 0, 0, 0);
            row[j] = 0;
            const int k = token(pass, j);
            if (there(k)) {
                const uint8_t* at = from.row(p.k, k);
                lo[j] = *(const uint4*)(at + 16 * mine.unit.c0);
                hi[j] = *(const uint4*)(at + 16 * mine.unit.c1);
                if (mine.unit.turned) row[j] = table_row(p, i + k);
            }
        }
#pragma unroll
        for (int j = 0; j < T; ++j) {
            float4 cs[4];
            if (mine.unit.turned) {
                const float4* at = p.table + (int64_t)row[j] * (p.rot >> 2) + 4 * mine.u;
#pragma unroll
                for (int e = 0; e < 4; ++e) cs[e] = at[e];
            }
            turn<BF16>(lo[j], hi[j], cs, mine.unit.turned, p.pairs, held[j]);
        }
    };
    auto passes = [&](bool again, auto each) {   // token by token, the rows loaded where they are not held
        for (int k = 0; k < n_pass; ++k) {
            if (again) load(k);
#pragma unroll
            for (int j = 0; j < T; ++j) each(token(k, j), held[j]);
        }
    };
    // smallest and largest of each channel; `strange` is a NaN once a value is none or infinite
    float low[16], high[16], strange = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) low[e] = kInf, high[e] = -kInf;
    passes(true, [&](int k, float (&f)[16]) {
        if (!there(k)) return;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            low[e] = fminf(low[e], f[e]);
            high[e] = fmaxf(high[e], f[e]);
            strange = __builtin_fmaf(f[e], 0.0f, strange);
        }
    });
    // the largest value, of the run's finite ones
    float largest = 0.0f;
    auto over_all = [&](float x) {
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) x = fmaxf(x, __shfl_xor(x, k, 64));
        return x;
    };
#pragma unroll
    for (int e = 0; e < 16; ++e) largest = fmaxf(largest, fmaxf(-low[e], high[e]));   // (-infinity where no token is)
    largest = over_all(strange != strange ? kInf : largest);
    const bool special = largest == kInf;
    if (special) {   // again: a NaN as 0, infinities beyond every finite value
        largest = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) low[e] = kInf, high[e] = -kInf;
        passes(true, [&](int k, float (&f)[16]) {
            if (!there(k)) return;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float x = f[e] != f[e] ? 0.0f : f[e];
                low[e] = fminf(low[e], x);
                high[e] = fmaxf(high[e], x);
                largest = fmaxf(largest, fabsf(x) < kInf ? fabsf(x) : 0.0f);
            }
        });
        largest = over_all(largest);
    }
    float s = largest < 0x1p-90f ? 0.0f : largest * (1.0f / kLargest);
    float grow = 1.0f;
    if (begin) {
        s = fmaxf(s, was);
        if (s > was) grow = was / s;
    }
    wave_sync();   // every lane has read the scale
    if (lane == 0) *sp = s;
    const float inv = s > 0.0f ? 1.0f / s : 0.0f;
    auto scaled = [&](float x) {
        const float y = x * inv;
        return !special || fabsf(x) < kInf ? y : x != x ? 0.0f : copysignf(kLargest, x);
    };
    passes(n_pass > 1, [&](int k, float (&f)[16]) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float four[4] = {scaled(f[4 * q]), scaled(f[4 * q + 1]), scaled(f[4 * q + 2]), scaled(f[4 * q + 3])};
            w[q] = near_codes<E4M3>(four);
        }
        if (!there(k)) return;
        uint8_t* at = codes + (begin + k) * d;
        *(uint2*)(at + 8 * mine.unit.c0) = make_uint2(w[0], w[1]);
        *(uint2*)(at + 8 * mine.unit.c1) = make_uint2(w[2], w[3]);
    });
    if (!p.boxes) {
        if (grow != 1.0f) before.rescale(grow, mine, [](auto&) {});
        return;
    }
    // The ends of the lane's channels as codes before they are rounded, those of the old tokens among them.  (A lane without a
    // token has infinity on either side.)
    if (!special) {
#pragma unroll
        for (int e = 0; e < 16; ++e) low[e] *= inv, high[e] *= inv;   // (infinity, or a NaN where inv is 0: neither is taken)
    } else if (there(mine.slot)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) low[e] = scaled(low[e]), high[e] = scaled(high[e]);
    }
    before.rescale(grow, mine, [&](auto& w) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f[OldKeys<E4M3>::kTurns][4];
#pragma unroll
            for (int t = 0; t < OldKeys<E4M3>::kTurns; ++t) codes_to_f32<E4M3>(w[t][q], f[t]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < OldKeys<E4M3>::kTurns; ++t) {
                    low[4 * q + e] = fminf(low[4 * q + e], f[t][e]);
                    high[4 * q + e] = fmaxf(high[4 * q + e], f[t][e]);
                }
        }
    });
    // The lanes of a unit together: a lane an end of a channel's range at a time.
    wave_sync();   // (the box of the run before is read)
#pragma unroll
    for (int e = 0; e < 16; ++e) s_box[e * kBoxRow + lane] = low[e], s_box[(16 + e) * kBoxRow + lane] = high[e];
    wave_sync();
    uint8_t* to = p.boxes + (page * a.heads + h) * 2 * (int64_t)d;
    const int half = p.rot >> 4, used_slots = min(mine.slots, max(len, begin));
    for (int v = lane; v < 2 * d; v += 64) {
        const bool upper = v >= d;
        const int ch = upper ? v - d : v, chunk = ch >> 3;
        const bool apart = !p.pairs && chunk < 2 * half;
        const int u = apart ? (chunk >= half ? chunk - half : chunk) : chunk >> 1;
        const int e = 8 * (apart ? chunk >= half : chunk & 1) + (ch & 7) + (upper ? 16 : 0);
        float x = upper ? -kInf : kInf;
        for (int t = 0; t < used_slots; t += 8)   // (eight reads at a time, none waiting for another)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = s_box[e * kBoxRow + min(t + j, used_slots - 1) * units + u];
                x = upper ? fmaxf(x, y) : fminf(x, y);
            }
        const float one[4] = {x, 0.0f, 0.0f, 0.0f};
        to[v] = (uint8_t)f32_to_codes<E4M3>(one);
    }
}

// Query rows: a lane one unit of kQHeads heads of a token, whose table entries it
// reads once.
constexpr int kQHeads = 4;

template <bool BF16>
__device__ __forceinline__ void turn_queries(const PageArgs& a, const AppendArgs& p, int64_t item)
{
    const int64_t at = item * 64 + (threadIdx.x & 63);
    if (at >= p.q_lanes) return;
    const uint32_t units = a.d >> 4;
    const int64_t tg = (at >> 32) ? at / units : (uint32_t)at / units;
    const int u = (int)(at - tg * units);
    const int64_t i = (tg >> 32) ? tg / p.q_groups : (uint32_t)tg / (uint32_t)p.q_groups;
    const int h0 = (int)(tg - i * p.q_groups) * kQHeads;
    if (p.rot && p.positions[i] < 0 && a.slots[i] < 0) return;   // no row of a request
    const Unit unit = unit_of(p, u);
    float4 cs[4];
    if (unit.turned) {
        const float4* t = p.table + (int64_t)table_row(p, i) * (p.rot >> 2) + 4 * u;
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e] = t[e];
    }
    const uint8_t* in = RowsFrom(p.q, i, 0).at;
    uint8_t* out = RowsFrom(p.q_out, i, 0).at;
    uint4 lo[kQHeads], hi[kQHeads];
#pragma unroll
    for (int k = 0; k < kQHeads; ++k) {
        const uint8_t* row = in + 2 * (int64_t)min(h0 + k, p.q_heads - 1) * p.q.stride_head;
        lo[k] = *(const uint4*)(row + 16 * unit.c0);
        hi[k] = *(const uint4*)(row + 16 * unit.c1);
    }
#pragma unroll
    for (int k = 0; k < kQHeads; ++k) {
        if (h0 + k >= p.q_heads) break;
        float f[16];
        turn<BF16>(lo[k], hi[k], cs, unit.turned, p.pairs, f);
        uint8_t* row = out + 2 * (int64_t)(h0 + k) * p.q_out.stride_head;
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = f32_to_row2(f[2 * e], f[2 * e + 1], BF16);
        *(uint4*)(row + 16 * unit.c0) = make_uint4(w[0], w[1], w[2], w[3]);
        *(uint4*)(row + 16 * unit.c1) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// A wave a window of rows and head, of K or of V, then waves for the query rows.  What
// bounds many rows is memory, where the K and V waves do not keep enough loads under way:
// 32,768 tokens, 8 KV heads and 32 query heads of 128, 182 us (756 MB, 4.2 TB/s), 106 of them
// for the K/V rows alone and the store without rotation and boxes 49.  (Tried where it took 178:
// the two kinds of blocks in turn 183; a block of four waves a run of keys 191, and a token of
// each of 1024 requests 94 us instead of 53.)
template <bool E4M3, bool BF16>
__global__ __launch_bounds__(kThreads, 3) void page_append_kernel(PageArgs a, AppendArgs p)
{
    __shared__ float s_box[kWaves][32 * kBoxRow];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
    if (item >= p.store_items) {
        if (p.q_lanes) turn_queries<BF16>(a, p, item - p.store_items);
        return;
    }
    const bool values = item & 1;
    const uint32_t hw = (uint32_t)(item >> 1);   // at most 2^31 windows x heads
    const int h = (int)(hw % (uint32_t)a.heads);
    const int64_t w0 = (int64_t)(hw / (uint32_t)a.heads) * p.window;
    const int64_t pool = a.n_pages * a.page;
    unsigned long long begins = run_begins(a, w0, p.window, [&](int64_t i, int64_t slot) {
        if (!p.n_bad || h || values) return;
        const int64_t pos = p.rot ? p.positions[i] : 0;
        if (slot >= pool || (p.rot && (pos >= p.n_pos || (pos < 0 && slot >= 0)))) atomicAdd(p.n_bad, 1u);
    });
    while (begins) {
        const int64_t i = w0 + __builtin_ctzll(begins);
        begins &= begins - 1;
        const int64_t slot = a.slots[i];
        const int64_t page = slot / a.page;
        const int begin = (int)(slot - page * a.page);
        const int len = run_length(a, i, slot, begin);
        if (values)
            store_run<E4M3, BF16>(a, p.v, true, i, h, page, begin, len);
        else
            append_keys<E4M3, BF16>(a, p, s_box[wave], i, h, page, begin, len);
    }
}

}  // namespace
}  // namespace fkv

using namespace fkv;

extern "C" int fkv_page_append(const fkv_page_desc* desc, const fkv_rotate_desc* rotate, const fkv_row_desc* rows_q,
                               const fkv_row_desc* rows_q_out, const fkv_row_desc* rows_k, const fkv_row_desc* rows_v,
                               const void* q_rows, void* q_out, const void* k_rows, const void* v_rows, int64_t n_tokens,
                               const int64_t* slots, const int32_t* positions, const float* table, uint8_t* k_codes,
                               uint8_t* v_codes, float* scales, uint8_t* boxes, uint32_t* n_bad, void* stream)
{
    if (!page_desc_ok(desc) || !row_desc_ok(rows_k) || !row_desc_ok(rows_v) || rows_k->type != rows_v->type || n_tokens < 0 ||
        n_tokens > kMostRows)
        return FKV_ERR_INVALID_ARG;
    const int32_t rot = rotate ? rotate->rot : 0;
    if (rotate && (rot < 0 || rot > desc->d || rot % 16 || (rotate->pairing != FKV_ROTATE_HALVES && rotate->pairing != FKV_ROTATE_PAIRS) ||
                   (rot && (rotate->n_pos < 1 || rotate->n_pos > ((int64_t)1 << 31) || !table || !aligned(table, 16)))))
        return FKV_ERR_INVALID_ARG;
    const bool with_q = q_rows != nullptr;
    if (with_q != (q_out != nullptr)) return FKV_ERR_INVALID_ARG;
    if (with_q && (!rotate || rotate->q_heads < 1 || rotate->q_heads > 65535 || !row_desc_ok(rows_q) || !row_desc_ok(rows_q_out) ||
                   rows_q->type != rows_k->type || rows_q_out->type != rows_k->type || !aligned(q_rows, 16) || !aligned(q_out, 16)))
        return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8) ||
        !aligned(boxes, 16) || !aligned(n_bad, 4))
        return FKV_ERR_INVALID_ARG;
    if (n_tokens == 0) return FKV_OK;
    if (!k_rows || !v_rows || !slots || !aligned(k_rows, 16) || !aligned(v_rows, 16) || !aligned(slots, 8) ||
        (rot && (!positions || !aligned(positions, 4))))
        return FKV_ERR_INVALID_ARG;
    const PageArgs a = {k_codes, v_codes, (float2*)scales, slots, n_tokens, desc->n_pages, desc->page, desc->heads, desc->d};
    AppendArgs p = {};
    p.q = rows_of(rows_q, q_rows), p.q_out = rows_of(rows_q_out, q_out);
    p.k = rows_of(rows_k, k_rows), p.v = rows_of(rows_v, v_rows);
    p.positions = positions, p.table = (const float4*)table, p.boxes = boxes, p.n_bad = n_bad;
    p.n_pos = rotate ? rotate->n_pos : 0;
    p.rot = rot;
    p.pairs = rotate && rotate->pairing == FKV_ROTATE_PAIRS;
    // As many rows a wave as leave four thousand waves, up to a page's worth: a wave writes the runs that begin among them one
    // by one, but waves of rows in which none begins hold up the others.  One row, and so many (us): 12 prompts of 2936 rows in
    // all, 8 heads of 80, 51 and 29; a token of each of 1024 requests, 8 heads of 128, 59 and 60; of 64 requests 32 tokens 56 and 35.
    const int64_t row_heads = n_tokens * desc->heads;
    p.window = (int32_t)std::min((int64_t)std::min(desc->page, 64), std::max((int64_t)1, (row_heads + 2047) / 2048));
    p.store_items = (n_tokens + p.window - 1) / p.window * desc->heads * 2;
    if (with_q) {
        p.q_heads = rotate->q_heads;
        p.q_groups = (p.q_heads + kQHeads - 1) / kQHeads;
        p.q_lanes = n_tokens * p.q_groups * (desc->d / 16);
    }
    const int64_t blocks = (p.store_items + (p.q_lanes + 63) / 64 + kWaves - 1) / kWaves;
    if (p.store_items > kMostBlocks || blocks > kMostBlocks) return FKV_ERR_UNSUPPORTED;
    const bool e4m3 = desc->format == FKV_PAGE_E4M3, bf16 = rows_k->type == FKV_ROW_BF16;
    auto kern = e4m3 ? bf16 ? page_append_kernel<true, true> : page_append_kernel<true, false>
                     : bf16 ? page_append_kernel<false, true> : page_append_kernel<false, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, p);
    return launch_status();
}
