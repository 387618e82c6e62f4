// page_rows_device.h -- what the kernels that write and read rows of the paged
// cache share: where rows lie, the exchange between the layouts of keys and
// values, and the writing of a run of rows.
#pragma once

#include "page_common.h"

namespace fkv {

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

constexpr int64_t kMostBlocks = 0x7fffff00;
constexpr int64_t kMostRows = (int64_t)1 << 40;   // beyond any memory; times the heads it is a number of 64 bits

inline Rows rows_of(const fkv_row_desc* r, const void* at)
{
    if (!at) return Rows{nullptr, 1, 0, 0, 0};
    return Rows{(uint8_t*)at, r->group, r->stride_group, r->stride_token, r->stride_head};
}

// A run: a row and those after it whose slots follow one another within a page.
// Of `window` rows from w0 on, those that begin one: at a page's first token, or
// where the row before does not lead up to them.  `each` is told every row's slot.
template <typename F>
__device__ __forceinline__ unsigned long long run_begins(const PageArgs& a, int64_t w0, int window, F each)
{
    const int lane = threadIdx.x & 63;
    const int64_t i = w0 + lane, pool = a.n_pages * a.page;
    bool first = false;
    if (lane < window && i < a.n_tokens) {
        const int64_t slot = a.slots[i], before = i ? a.slots[i - 1] : -2;
        first = slot >= 0 && slot < pool && ((uint32_t)(slot % a.page) == 0 || before != slot - 1);
        each(i, slot);
    }
    return __ballot(first);
}

// The rows of the run that begins with row i, at token `begin` of its page.
__device__ __forceinline__ int run_length(const PageArgs& a, int64_t i, int64_t slot, int begin)
{
    const int lane = threadIdx.x & 63;
    const int most = (int)min((int64_t)(a.page - begin), a.n_tokens - i);
    int len = 1;
    for (int base = 1; base < most; base += 64) {
        const bool follows = base + lane < most && a.slots[i + base + lane] == slot + base + lane;
        const unsigned long long m = __ballot(!follows);
        const int run = m ? __builtin_ctzll(m) : 64;
        len = base + run;
        if (run < 64) break;
    }
    return len;
}

template <bool E4M3>
__device__ __forceinline__ uint32_t grown(uint32_t w, float grow)   // four codes
{
    float f[4];
    codes_to_f32<E4M3>(w, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] *= grow;
    return f32_to_codes<E4M3>(f);
}

// A wave brings the codes that a page holds before `begin` to a new scale, times `grow`: 16 bytes
// a lane and turn -- of the keys' rows as they lie, of the values 16 tokens of a channel --
// kOldTurns turns in flight.  (One word a lane and turn, each turn waiting for its load: a token
// stored to each of 64 requests' pages of 64 tokens x 128 channels, 8 heads, whose scales grow
// took 17.6 us with the launch that set them back, so 12.0; of 4096 requests 407, so 232.  With the
// first ones read before the new scale is known 12.0 and 228, but where scales do not grow, as most
// do not, 8192 requests then take 309 us in place of 282.)
constexpr int kOldTurns = 4;

template <bool E4M3>
__device__ __forceinline__ void rescale_codes(uint8_t* codes, int d, bool values, int begin, float grow)
{
    const int n = values ? (begin + 15) / 16 * d : begin * (d / 16);   // 16-byte parts
    for (int t0 = threadIdx.x & 63; t0 < n; t0 += kOldTurns * 64) {
        uint4 held[kOldTurns];
#pragma unroll
        for (int t = 0; t < kOldTurns; ++t) held[t] = ((const uint4*)codes)[min(t0 + t * 64, n - 1)];
#pragma unroll
        for (int t = 0; t < kOldTurns; ++t) {
            const int at = t0 + t * 64;
            if (at >= n) break;
            const uint4 w = make_uint4(grown<E4M3>(held[t].x, grow), grown<E4M3>(held[t].y, grow), grown<E4M3>(held[t].z, grow),
                                       grown<E4M3>(held[t].w, grow));
            uint8_t* to = codes + (int64_t)at * 16;
            const int keep = values ? begin - at / d * 16 : 16;   // of the value tokens that `begin` lies among, only those before it
            if (keep >= 16) {
                *(uint4*)to = w;
                continue;
            }
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (keep >= 4 * q + 4) *(uint32_t*)(to + 4 * q) = words[q];
                else
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (keep > 4 * q + e) to[4 * q + e] = (uint8_t)(words[q] >> (8 * e));
            }
        }
    }
}

// A wave writes a run of one head's keys or values: len rows from row i on, to the
// tokens begin .. of a page.  Up to 64 columns of it (a page of 64 tokens x 128
// channels) are held in registers between the largest element and the codes; larger
// pages are read a second time (from the caches).  Rows are read 16 bytes a lane,
// codes written 8 (keys) and 16 (values) bytes a lane.  The largest element is found
// on the rows' bits, two at a time: without the sign they are in the order of the
// numbers, and what is not finite comes last; only a run that has such elements looks
// at each.
constexpr int kPasses = 4;   // of 16 columns

template <bool E4M3, bool BF16>
__device__ __forceinline__ void store_run(const PageArgs& a, const Rows& rows, bool values, int64_t i, int h, int64_t page, int begin, int len)
{
    typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
    constexpr uint32_t kInf = BF16 ? 0x7f80 : 0x7c00;
    constexpr float kLargest = E4M3 ? kLargestE4m3 : kLargestInt8;
    const int lane = threadIdx.x & 63, c16 = lane & 15, tq = lane >> 4;
    const uint32_t chunks = a.d / 8;
    const int end = begin + len;
    const int g0 = begin >> 4;
    const int columns = (((end + 15) >> 4) - g0) * chunks;
    const RowsFrom from(rows, i, h);
    float* sp = (float*)&a.scales[page * a.heads + h] + (values ? 1 : 0);
    uint8_t* codes = (values ? a.v_codes : a.k_codes) + (page * a.heads + h) * (int64_t)a.page * a.d;
    const float was = begin ? *sp : 0.0f;
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
    float s = largest < 0x1p-90f ? 0.0f : largest * (1.0f / kLargest);
    if (begin) {
        s = fmaxf(s, was);
        // (out of the way of runs that begin a page: 32,768 tokens with the rows in the caches 49 -> 45 us)
        if (__builtin_expect(s > was, 0)) rescale_codes<E4M3>(codes, a.d, values, begin, was / s);
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

}  // namespace fkv
