// page_attend_device.h -- what the kernels of attention over the paged cache share:
// what a request's rows see, where its keys lie, a wave's pass over the tiles of few
// rows, and the joining of the sums of several passes.
#pragma once

#include "page_common.h"

#include <type_traits>

namespace fkv {
namespace {

typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kTile = 64;          // keys of a tile
constexpr int kFewRows = 16;       // rows of the kernel for few rows
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kTop = 256.0f;     // the weight of a key at the reference maximum, and
constexpr float kSlack = 6.0f;     // how far scores may pass that before it moves: weights stay below 2^14 (of large scores the difference
                                   // is exact, and the sum of both might be rounded up to the score)
constexpr float kLeast = 0x1p-100f;
// Sums of weights times values that are to be joined with others are kept times 2^-30: bfloat16 values may be near
// fp32's end, where a sum of a few of them is beyond it and their mean is not (2^24 keys of weights up to 2^6).
constexpr float kPart = 0x1p-30f;

struct AttendArgs {
    const uint8_t* k_codes;
    const uint8_t* v_codes;
    const float2* scales;
    const uint8_t* q;
    uint8_t* out;
    float* lse;
    const int32_t* tables;
    const int32_t* kv_len;
    const int32_t* q_start;
    const float* slopes;
    const int32_t* prefix;
    const int32_t* first;
    float* part;    // [row][split][d] sums of a split's weights times values, times kPart, or [piece][2][row][d]
    float2* stat;   // likewise: their maximum and sum of weights
    int2* pieces;   // [request][KV head] how many pieces of the line its tiles lie in, and the first
    int64_t n_req, n_tokens, max_new, max_kv, max_pages, n_pages;
    int64_t q_token, q_head, o_token, o_head;
    int32_t page, heads, group, d, window, sinks;
    int32_t bf16, causal;
    int32_t n_splits, split_tiles;
    const int32_t* listed;   // [token][KV head][n_listed] columns of the token's block table, of attention to listed pages
    int64_t n_listed;
    int64_t searched;      // rows of q whose requests the kernels for lists look up (0: max_new places a request)
    int32_t piece_rows;    // of a KV head: max_new x group
    uint32_t per_page;     // 16-key groups of a page
    uint32_t per_page_inv; // and their reciprocal, 2^32 / per_page rounded up (0: one)
    float scale, softcap;
};

// A request as a block sees it.
struct Request {
    int kv, rows, start, pos0;   // keys; query tokens, the first one's row and position
};

__device__ __forceinline__ Request request_of(const AttendArgs& a, int64_t r)
{
    Request q;
    const int64_t most = min(a.max_kv, a.max_pages * a.page);
    q.kv = (int)min((int64_t)max(a.kv_len[r], 0), most);
    const int64_t b = min(max((int64_t)a.q_start[r], (int64_t)0), a.n_tokens);
    const int64_t e = min(max((int64_t)a.q_start[r + 1], b), a.n_tokens);
    q.start = (int)b;
    q.rows = (int)min(e - b, a.max_new);
    q.pos0 = q.kv - (int)(e - b);
    return q;
}

// Prompts and single tokens in one call leave most of n_req x max_new places empty.  Then
// a launch has a place for each row of q, and finds its request: the last whose rows
// begin at `index` or before.  PER rows a place: of a request's rows the places
// start / PER + r on, which are enough for any rows before the next request's.  -1: none.
// (A step of 30 single tokens, 2048 of a chunk and 33 more, 8 heads of 128: selection 208 -> 73 us, attention to lists
// 987 -> 640.)
__device__ __forceinline__ int64_t first_place(const AttendArgs& a, int64_t r, int per)
{
    const uint32_t start = (uint32_t)min(max((int64_t)a.q_start[r], (int64_t)0), a.n_tokens);
    return per == 1 ? start : start / (uint32_t)per + r;
}

__device__ __forceinline__ int64_t request_at(const AttendArgs& a, int64_t index, int per)
{
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, end = a.n_req;   // the requests not settled; but for the first round lo's rows begin early enough
    for (;;) {
        const int64_t step = (end - lo + 63) >> 6, j = lo + lane * step;
        const int n = __builtin_popcountll(__ballot(j < end && first_place(a, min(j, end - 1), per) <= index));
        if (n == 0) return -1;
        lo += (n - 1) * step;
        if (step == 1) return lo;
        end = min(end, lo + step);
    }
}

// What token i of a request sees: keys [lo, hi), of those below wlo only the
// sinks.
struct Seen {
    int lo, hi, wlo;
};

__device__ __forceinline__ Seen seen_of(const AttendArgs& a, const Request& rq, int64_t r, int i)
{
    const int pos = rq.pos0 + i;
    Seen s;
    s.lo = a.first ? max(a.first[rq.start + i], 0) : 0;
    s.hi = rq.kv;
    if (a.causal) s.hi = min(rq.kv, max(pos + 1, a.prefix ? max(a.prefix[r], 0) : 0));
    s.wlo = a.window ? pos - a.window + 1 : 0;
    return s;
}

// The tiles that some row of a block sees: s0 .. s0+ns-1 (sinks), then w0 ..,
// n in all; and what every row sees of all tiles.
struct Tiles {
    int s0, ns, w0, n;
    int lo, hi, wlo;   // a tile in [lo, hi) that lies above wlo or below the sinks needs no mask
    __device__ __forceinline__ int tile(int e) const { return e < ns ? s0 + e : w0 + e - ns; }
};

__device__ __forceinline__ Tiles tiles_of(const AttendArgs& a, int lo_min, int lo_max, int hi_min, int hi_max, int wlo_min, int wlo_max)
{
    Tiles t;
    const int end = (hi_max + kTile - 1) / kTile;
    t.s0 = lo_min / kTile;
    t.ns = 0;
    t.w0 = t.s0;
    if (a.window) {
        t.w0 = max(lo_min, max(wlo_min, 0)) / kTile;
        const int s1 = min((int)((min((int64_t)a.sinks, (int64_t)hi_max) + kTile - 1) / kTile), t.w0);
        t.ns = max(0, s1 - t.s0);
    }
    t.n = t.ns + max(0, end - t.w0);
    t.lo = lo_max;
    t.hi = hi_min;
    t.wlo = wlo_max;
    return t;
}

__device__ __forceinline__ bool tile_whole(const AttendArgs& a, const Tiles& t, int j0)
{
    return j0 >= t.lo && j0 + kTile <= t.hi && (!a.window || j0 >= t.wlo || j0 + kTile <= a.sinks);
}

__device__ __forceinline__ bool visible(const AttendArgs& a, const Seen& s, int j)
{
    // (no branches: a select for each key)
    return (j >= s.lo) & (j < s.hi) & ((a.window == 0) | (j >= s.wlo) | (j < a.sinks));
}

// Loads of addresses that are the same in every lane, through the scalar cache:
// of arrays that no kernel here writes while it reads them.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p)
{
    return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// One of four by its number, through selects.
__device__ __forceinline__ int64_t one_of(int k, int64_t a, int64_t b, int64_t c, int64_t d)
{
    const bool odd = k & 1;
    const int64_t lo = odd ? b : a, hi = odd ? d : c;
    return k & 2 ? hi : lo;
}

// Where a request's 16-key group lies: its page and the group within it.  A
// group with no valid page is not there; it is given page 0, so that loads need
// no condition, and what they bring is masked.
struct Place {
    int id, in_page;
    bool here;
};

__device__ __forceinline__ Place place_of(const AttendArgs& a, const int32_t* table, int kv, int grp)
{
    Place p;
    p.here = grp * 16 < kv;
    grp = min(grp, (kv - 1) >> 4);   // kv >= 1
    const int at = a.per_page_inv ? (int)__umulhi((uint32_t)grp, a.per_page_inv) : grp;
    p.in_page = grp - at * (int)a.per_page;
    p.id = table[at];
    return p;
}

__device__ __forceinline__ void check_place(const AttendArgs& a, Place& p)
{
    p.here = p.here && (uint32_t)p.id < (uint64_t)a.n_pages;
    p.id = p.here ? p.id : 0;
}

// 16 codes to binary16, exact.  An int8 code c becomes 1024 + (c + 128) by
// placing the byte under the exponent of 1024, and 1152 less is c.
template <bool E4M3>
__device__ __forceinline__ half2_t codes2(uint32_t w, bool hi)
{
    if (E4M3) return hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w ^ 0x80808080u, hi ? 0x04030402u : 0x04010400u);
    const half2_t bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    return __builtin_bit_cast(half2_t, u) - bias;
}

template <bool E4M3>
__device__ __forceinline__ half8_t codes8(uint32_t a, uint32_t b)
{
    const half2_t p = codes2<E4M3>(a, false), q = codes2<E4M3>(a, true);
    const half2_t r = codes2<E4M3>(b, false), s = codes2<E4M3>(b, true);
    return half8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// Keeps the first n bytes of four words.
__device__ __forceinline__ uint4 first_bytes(uint4 w, int n)
{
    auto keep = [&](uint32_t x, int k) { return k >= 4 ? x : k <= 0 ? 0u : x & ((1u << (8 * k)) - 1u); };
    return make_uint4(keep(w.x, n), keep(w.y, n - 4), keep(w.z, n - 8), keep(w.w, n - 12));
}

// A bfloat16 row's power of two, from its largest element: largest * 2^e lies
// in [2^13, 2^14).  0 for a row of zeros and for one with no finite largest.
__device__ __forceinline__ int row_shift(float largest)
{
    const int ex = (int)((__float_as_uint(largest) >> 23) & 0xff);
    return ex == 0 || ex == 0xff ? 0 : min(max(127 + 13 - ex, -120), 120);
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// 8 elements of a q row to binary16.
__device__ __forceinline__ half8_t q8(uint4 w, bool bf16, float mul)
{
    if (!bf16) return __builtin_bit_cast(half8_t, w);
    half8_t h;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)(row_to_f32(u[e >> 1], e & 1, true) * mul);
    return h;
}

__device__ __forceinline__ float abs_most8(uint4 w)
{
    float m = 0.0f;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(row_to_f32(u[e >> 1], e & 1, true)));
    return m;
}

// Over the two halves of a wave, and over its four rows of 16 lanes: each
// lane gets the result of the lanes that share its lower bits.
__device__ __forceinline__ float halves_max(float a)
{
    const uint32_t u = __float_as_uint(a);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float halves_sum(float a)
{
    const uint32_t u = __float_as_uint(a);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float rows_max(float a)
{
    const uint32_t u = __float_as_uint(a);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

__device__ __forceinline__ float rows_sum(float a)
{
    const uint32_t u = __float_as_uint(a);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// cap * tanh(x / cap) in base 2, u being twice the tanh's argument in base 2:
// tanh t = 1 - 2 / (1 + e^2t).  For small t that is the difference of two numbers
// near 1, so the error is of the size of the cap, about 2^-23 of it: a score's is
// about 2^-16 for the caps up to kSmallCap that take this form.
constexpr float kSmallCap = 128.0f;

__device__ __forceinline__ float capped(float u, float cap)
{
    const float e = __builtin_amdgcn_exp2f(u);
    return cap * (1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + e));
}

// The same of a larger cap, x being the score in base 2: below |t| = 0.4 the series
// x (1 - t^2 / 3 + 2 t^4 / 15 - ..) to t^10, which ends within 2^-24 of itself, and the
// form above beyond, where its error is 2^-21 of the result.
__device__ __forceinline__ float capped_large(float x, float cap, float inv_cap)
{
    const float t = x * inv_cap, q = t * t;
    float p = __builtin_fmaf(q, -1382.0f / 155925.0f, 62.0f / 2835.0f);
    p = __builtin_fmaf(q, p, -17.0f / 315.0f);
    p = __builtin_fmaf(q, p, 2.0f / 15.0f);
    p = __builtin_fmaf(q, p, -1.0f / 3.0f);
    return fabsf(t) < 0.4f ? __builtin_fmaf(x * q, p, x) : capped(t * (2.0f * kLog2e), cap);
}

// ------------------------------------------------------------- few rows --

// One KV head of a request and at most 16 rows (query tokens x heads of the
// group): what bounds it is the reading of the codes, 2 d bytes a key.  Codes go
// from memory to registers in the operands' own layout, 16 bytes a lane and
// load, the next tile's keys while a tile's softmax runs.
// The left operand of S^T takes row t*4+i of key group g as its row 4g+i in
// product t, so that lane group g ends up with keys 16g .. 16g+15, which are the
// 16 bytes of a value channel that it loads.  NC: chunks of 64 channels.
__device__ __forceinline__ Tiles few_tiles(const AttendArgs& a, const Request& rq, int64_t r)
{
    int lo_min = 0x7fffffff, lo_max = 0, hi_min = 0x7fffffff, hi_max = 0, wlo_min = 0x7fffffff, wlo_max = 0;
    for (int i = 0; i < rq.rows; ++i) {
        const Seen s = seen_of(a, rq, r, i);
        lo_min = min(lo_min, s.lo), lo_max = max(lo_max, s.lo);
        hi_min = min(hi_min, s.hi), hi_max = max(hi_max, s.hi);
        wlo_min = min(wlo_min, s.wlo), wlo_max = max(wlo_max, s.wlo);
    }
    return tiles_of(a, lo_min, lo_max, hi_min, hi_max, wlo_min, wlo_max);
}

// A wave's rows: this lane's is number row of the block's, token tok of the
// request, query head head.
struct FewRow {
    int row, tok, head;
};

__device__ __forceinline__ FewRow few_row(const AttendArgs& a, const Request& rq, int h)
{
    FewRow w;
    w.row = min((int)threadIdx.x & 15, rq.rows * a.group - 1);
    w.tok = w.row / a.group;
    w.head = h * a.group + w.row % a.group;
    return w;
}

// Statistics and sums of a wave: lane 16g + c holds channels 16t + 4g .. + 3 of
// row c in acc[t], times 2^8 / vref.
template <int NC>
struct FewSums {
    float m, l, vref;
    float4_t acc[4 * NC];
    __device__ __forceinline__ FewSums() : m(-__builtin_inff()), l(0.0f), vref(kLeast)
    {
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) acc[t] = float4_t{0, 0, 0, 0};
    }
};

// What a lane knows of its row: the right operand of S^T -- channels 64c + 16g .. + 15
// -- and how its scores are formed.
template <int NC>
struct FewQuery {
    half8_t qf[NC][2];
    float mul, cap, cap2, slope2;
    int pos;
    bool large_cap, slopes;
    __device__ __forceinline__ FewQuery(const AttendArgs& a, const Request& rq, const FewRow& fr)
    {
        const int g = (threadIdx.x & 63) >> 4;
        const uint8_t* qp = a.q + 2 * ((int64_t)(rq.start + fr.tok) * a.q_token + fr.head * a.q_head);
        int shift = 0;
        uint4 w[NC][2];
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e = c * 64 + g * 16;
            w[c][0] = w[c][1] = make_uint4(0, 0, 0, 0);
            if (e < a.d) w[c][0] = *(const uint4*)(qp + 2 * e), w[c][1] = *(const uint4*)(qp + 2 * e + 16);
            if (a.bf16) most = fmaxf(most, fmaxf(abs_most8(w[c][0]), abs_most8(w[c][1])));
        }
        if (a.bf16) shift = row_shift(rows_max(most));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            qf[c][0] = q8(w[c][0], a.bf16, pow2(shift));
            qf[c][1] = q8(w[c][1], a.bf16, pow2(shift));
        }
        cap = a.softcap;
        cap2 = a.softcap * kLog2e;
        large_cap = a.softcap > kSmallCap;
        mul = pow2(-shift) * (a.softcap > 0.0f && !large_cap ? a.scale * 2.0f * kLog2e / a.softcap : a.scale * kLog2e);
        slopes = a.slopes != nullptr;
        slope2 = slopes ? a.slopes[fr.head] * kLog2e : 0.0f;
        pos = rq.pos0 + fr.tok;
    }
};

// The products of a tile's keys with the row: of keys j0g .. j0g+15 in turn, before
// their factors.
template <bool E4M3, int NC>
__device__ __forceinline__ void few_products(const uint4 (&kw)[4][NC], const FewQuery<NC>& q, float4_t (&s)[4])
{
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        s[t] = float4_t{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<E4M3>(kw[t][c].x, kw[t][c].y), q.qf[c][0], s[t], 0, 0, 0);
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<E4M3>(kw[t][c].z, kw[t][c].w), q.qf[c][1], s[t], 0, 0, 0);
        }
    }
}

// The tile's scores, weights and values into the sums.  sc: the scales of the lane's key
// group, which is there (`here`) or not; vw: its values.
template <bool E4M3, int NC>
__device__ __forceinline__ void few_update(const AttendArgs& a, const Request& rq, const Seen& mine, const FewQuery<NC>& q, FewSums<NC>& st,
                                           const float4_t (&s)[4], uint4 (&vw)[4 * NC], float2 sc, bool here, bool mask, int j0g)
{
    const float mulk = q.mul * sc.x;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = s[i >> 2][i & 3] * mulk;
    if (q.large_cap) {
        const float inv = 1.0f / q.cap2;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = capped_large(x[i], q.cap2, inv);
    } else if (q.cap > 0.0f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = capped(x[i], q.cap2);
    }
    if (q.slopes) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] -= q.slope2 * fabsf((float)(j0g + i - q.pos));
    }
    if (mask) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!here || !visible(a, mine, j0g + i)) x[i] = -__builtin_inff();
        if (E4M3) {   // codes after the last key may be anything, a NaN among it
            const int n = here ? rq.kv - j0g : 0;
#pragma unroll
            for (int t = 0; t < 4 * NC; ++t) vw[t] = first_bytes(vw[t], n);
        }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
    const float vtop = top > -__builtin_inff() ? sc.y : 0.0f;   // of a group of which the row sees a key
    top = rows_max(top);
    if (__any(top - st.m > kSlack || vtop > st.vref)) {
        const float vnew = rows_max(fmaxf(st.vref, vtop));
        const float mnew = fmaxf(st.m, top);
        const float shrink = mnew == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(st.m - mnew);
        st.l *= shrink;
        const float k = shrink * (st.vref / vnew);
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) st.acc[t] *= k;
        st.m = mnew;
        st.vref = vnew;
    }
    const float m0 = st.m == -__builtin_inff() ? 0.0f : st.m;
    const float vs = fminf(sc.y * (kTop / st.vref), kTop);   // (beyond that only where all weights are 0)
    half8_t p[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(x[i] - m0);
        st.l += w;
        p[i >> 3][i & 7] = (_Float16)(w * vs);
    }
#pragma unroll
    for (int t = 0; t < 4 * NC; ++t) {
        st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<E4M3>(vw[t].x, vw[t].y), p[0], st.acc[t], 0, 0, 0);
        st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<E4M3>(vw[t].z, vw[t].w), p[1], st.acc[t], 0, 0, 0);
    }
}

// A wave over tiles e0, e0 + step, .. below e1 (one at least).
template <bool E4M3, int NC>
__device__ __forceinline__ void few_keys(const AttendArgs& a, const Request& rq, int64_t r, int h, const Tiles& tl, const FewRow& fr,
                                         int e0, int step, int e1, FewSums<NC>& st)
{
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int d = a.d;
    const int64_t per_head = (int64_t)a.page * d;
    const Seen mine = seen_of(a, rq, r, fr.tok);
    const int32_t* table = a.tables + r * a.max_pages;
    const int gk = c16 >> 2;   // the key group of this lane's left-operand rows
    // channels beyond d are loaded from the last ones: q is zero there, and their sums go nowhere
    int kc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) kc[c] = (c16 & 3) * d + min(c * 64 + g * 16, d - 16);
    const uint8_t* k_head = a.k_codes + h * per_head;
    const uint8_t* v_head = a.v_codes + h * per_head + c16 * 16;
    const int64_t per_id = a.heads * per_head;
    const float2* scale_head = a.scales + h;
    uint4 kw[4][NC];
    float2 sc, sc_next;
    auto load_keys = [&](const Place& p) {
        const uint8_t* kp = k_head + p.id * per_id + p.in_page * 16 * d;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) kw[t][c] = *(const uint4*)(kp + kc[c] + t * 4 * d);
    };
    int j0 = tl.tile(e0) * kTile;
    Place pk = place_of(a, table, rq.kv, (j0 >> 4) + gk), pv = place_of(a, table, rq.kv, (j0 >> 4) + g);
    int j1 = tl.tile(min(e0 + step, e1 - 1)) * kTile;
    Place pk1 = place_of(a, table, rq.kv, (j1 >> 4) + gk), pv1 = place_of(a, table, rq.kv, (j1 >> 4) + g);
    check_place(a, pk);
    check_place(a, pv);
    load_keys(pk);
    sc = scale_head[(int64_t)pv.id * a.heads];

    const FewQuery<NC> query(a, rq, fr);

    for (int e = e0; e < e1; e += step) {
        // the tile's values, on their way while its scores are formed
        uint4 vw[4 * NC];
        const uint8_t* vp = v_head + pv.id * per_id + pv.in_page * 16 * d;
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) vw[t] = *(const uint4*)(vp + min(t * 16, d - 16) * 16);
        const bool here = pv.here;
        const bool mask = !tile_whole(a, tl, j0) || __any(!here);
        const int j0g = j0 + g * 16;
        if (!here) sc = make_float2(0.0f, 0.0f);
        float4_t s[4];
        few_products<E4M3>(kw, query, s);
        // the next tile's keys, and the pages of the one after
        if (e + step < e1) {
            check_place(a, pk1);
            check_place(a, pv1);
            load_keys(pk1);
            sc_next = scale_head[(int64_t)pv1.id * a.heads];
            j0 = j1, pv = pv1;
            j1 = tl.tile(min(e + 2 * step, e1 - 1)) * kTile;
            pk1 = place_of(a, table, rq.kv, (j1 >> 4) + gk);
            pv1 = place_of(a, table, rq.kv, (j1 >> 4) + g);
        }
        few_update<E4M3>(a, rq, mine, query, st, s, vw, sc, here, mask, j0g);
        sc = sc_next;
    }
    st.l = rows_sum(st.l);
}

// ----------------------------------------------------------------- join --

// The splits of a row together: weights 2^(m_s - max m).  R waves of a block
// take one row's splits in turn (R = 1: a row each); a lane holds four channels
// of every second split of its wave (of each, where d > 128), and the sums of
// kJoin splits are on their way at a time.  128 rows of about 58 splits each: 5 us,
// most of it the launch and two dependent reads.
constexpr int kJoin = 4;
constexpr int kManySplits = 32;   // from which on a block takes one row

template <int R>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a)
{
    __shared__ float4_t s_o[kWaves][64];
    __shared__ float s_l[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t q_heads = (int64_t)a.heads * a.group;
    const int64_t item = R == 1 ? (int64_t)blockIdx.x * kWaves + wave : blockIdx.x;
    const int64_t index = item / q_heads, hq = item % q_heads;
    if (index >= (a.searched ? a.searched : a.n_req * a.max_new)) return;
    const int64_t r = a.searched ? request_at(a, index, 1) : index / a.max_new;
    if (r < 0) return;
    const Request rq = request_of(a, r);
    const int64_t i = a.searched ? index - rq.start : index % a.max_new;
    if (i < 0 || i >= rq.rows) return;   // (negative: of starts out of order)
    const int2 piece = a.pieces ? a.pieces[r * a.heads + hq / a.group] : make_int2(a.n_splits, 0);
    const int n = piece.x;
    if (a.pieces && n == 1) return;   // written already
    const int64_t token = rq.start + i;
    // where split s lies: the first piece's sums in its second place, the others' in their first
    const int64_t at = a.pieces ? 2 * (int64_t)piece.y * a.piece_rows + i * a.group + hq % a.group : (token * q_heads + hq) * a.n_splits;
    const int64_t per_split = a.pieces ? 2 * a.piece_rows : 1, of_first = a.pieces ? a.piece_rows : 0;
    auto place = [&](int s) { return at + s * per_split + (s ? 0 : of_first); };
    float mm = -__builtin_inff();
    for (int s = lane; s < n; s += 64) mm = fmaxf(mm, a.stat[place(s)].x);
    mm = halves_max(mm);
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) mm = fmaxf(mm, __shfl_xor(mm, k, 64));
    const float m0 = mm == -__builtin_inff() ? 0.0f : mm;
    const bool wide = a.d > 128;
    const int sub = wide ? 0 : lane >> 5, subs = wide ? 1 : 2, q4 = wide ? lane : lane & 31;
    const bool has = 4 * q4 < a.d;
    const int first = (R == 1 ? 0 : wave * subs) + sub, step = R * subs;
    float ll = 0.0f;
    float4_t o = {0, 0, 0, 0};
    for (int s0 = first; s0 < n; s0 += kJoin * step) {
        float4_t p[kJoin];
        float2 st[kJoin];
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
            const int s = s0 + k * step;
            st[k] = make_float2(-__builtin_inff(), 0.0f);
            p[k] = float4_t{0, 0, 0, 0};
            if (s < n) {
                st[k] = a.stat[place(s)];
                if (has) p[k] = *(const float4_t*)(a.part + place(s) * a.d + 4 * q4);
            }
        }
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
            const float f = __builtin_amdgcn_exp2f(st[k].x - m0);
            ll += f * st[k].y;
            o += f * p[k];
        }
    }
    if (!wide) {
        ll = halves_sum(ll);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = halves_sum(o[e]);
    }
    if (R > 1) {
        s_o[wave][lane] = o;
        if (lane == 0) s_l[wave] = ll;
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) o += s_o[w][lane], ll += s_l[w];
    }
    const float inv = ll == 0.0f ? 0.0f : (1.0f / kPart) / ll;
    if (has && sub == 0)
        *(uint2*)(a.out + 2 * (token * a.o_token + hq * a.o_head + 4 * q4)) =
            make_uint2(f32_to_row2(o[0] * inv, o[1] * inv, a.bf16), f32_to_row2(o[2] * inv, o[3] * inv, a.bf16));
    if (lane == 0 && a.lse) a.lse[token * q_heads + hq] = ll == 0.0f ? -__builtin_inff() : kLn2 * (mm + __log2f(ll));
}

// ----------------------------------------------------------------- host --

inline bool attend_ok(const fkv_page_desc* p, const fkv_attend_desc* t)
{
    constexpr int64_t kMost = 1 << 30;
    return page_desc_ok(p) && t && t->n_req >= 0 && t->n_req <= kMost && t->n_tokens >= 0 && t->n_tokens <= kMost &&
           t->max_new >= 1 && t->max_new <= kMost && t->max_kv >= 0 && t->max_kv <= kMost && t->max_pages >= 1 &&
           t->max_pages <= (1 << 26) && stride_ok(t->q_stride_token) && stride_ok(t->q_stride_head) &&
           stride_ok(t->o_stride_token) && stride_ok(t->o_stride_head) && t->q_heads >= 1 && t->q_heads <= 65535 &&
           t->q_heads % p->heads == 0 && (t->type == FKV_ROW_F16 || t->type == FKV_ROW_BF16) &&
           t->scale - t->scale == 0.0f && t->softcap >= 0.0f && t->softcap - t->softcap == 0.0f &&
           (t->causal == 0 || t->causal == 1) && t->window >= 0 && t->window <= kMost && t->sinks >= 0 && t->sinks <= kMost;
}

// The arguments of a call that are alike in all kernels.
inline AttendArgs attend_args(const fkv_page_desc* desc, const fkv_attend_desc* attend, const uint8_t* k_codes, const uint8_t* v_codes,
                              const float* scales, const void* q, const int32_t* tables, const int32_t* kv_len,
                              const int32_t* q_start, const float* slopes, const int32_t* prefix, const int32_t* first, void* out,
                              float* lse)
{
    AttendArgs a = {};
    a.k_codes = k_codes, a.v_codes = v_codes, a.scales = (const float2*)scales;
    a.q = (const uint8_t*)q, a.out = (uint8_t*)out, a.lse = lse;
    a.tables = tables, a.kv_len = kv_len, a.q_start = q_start;
    a.slopes = slopes, a.prefix = prefix, a.first = first;
    a.n_req = attend->n_req, a.n_tokens = attend->n_tokens, a.max_new = attend->max_new, a.max_kv = attend->max_kv;
    a.max_pages = attend->max_pages, a.n_pages = desc->n_pages;
    a.q_token = attend->q_stride_token, a.q_head = attend->q_stride_head;
    a.o_token = attend->o_stride_token, a.o_head = attend->o_stride_head;
    a.page = desc->page, a.heads = desc->heads, a.group = attend->q_heads / desc->heads, a.d = desc->d;
    a.window = attend->window, a.sinks = attend->sinks;
    a.bf16 = attend->type, a.causal = attend->causal;
    a.per_page = (uint32_t)(desc->page / 16);
    a.per_page_inv = a.per_page == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + a.per_page - 1) / a.per_page);
    a.scale = attend->scale, a.softcap = attend->softcap;
    return a;
}

// The workspace: sums, then maxima and sums of weights, then the heads' pieces of the line.
struct Workspace {
    size_t stat, pieces, bytes;
};

}  // namespace
}  // namespace fkv
