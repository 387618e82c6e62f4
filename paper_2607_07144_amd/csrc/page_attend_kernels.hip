// page_attend_kernels.hip -- attention over the paged 8-bit cache, for gfx950.
//
// One pass over the keys with the running maximum and sum of a softmax, in base
// 2: with x the scores times log2 e,
//     m' = max(m, max x),  l' = l 2^(m-m') + sum 2^(x-m'),
//     o' = o 2^(m-m') + sum 2^(x-m') v.
// Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T, on
// matrix cores: the accumulator of S^T then holds one row's scores per lane
// (the lane's column), so the statistics are per-lane values, and the weights
// are already where the second product wants its right operand, with no way
// through shared memory -- the order in which a product sums over keys is
// free, so the keys are dealt to the accumulator's rows such that each lane
// ends up with consecutive ones.
//
// int8 codes and 8-bit floats are exact in binary16, and so is q (a bfloat16
// row is taken times a power of two that brings its largest element near 2^13;
// elements 2^27 times smaller than that round).  Key scales multiply the fp32
// scores.  Value scales differ from page to page, so they multiply the fp32
// weights before those are rounded to binary16: w = p * vs * 2^8 / vr with vr
// the largest value scale so far of what the row sees, so that w keeps its 11
// bits down to p vs / vr = 2^-22; the accumulators carry the factor 2^8 / vr.  m
// need not be the maximum itself: it moves, and the accumulators with it, only
// when a score passes it by more than 6, where w would near binary16's end.  Powers
// of two, logarithms and the
// reciprocals in a cap and in a value scale's share of the sum are the hardware's
// instructions, within about one unit of fp32's last place: far below the weights'
// 2^-11.
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
constexpr float kSlack = 6.0f;     // how far scores may pass that before it moves: weights stay below 2^14
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

// A wave over tiles e0, e0 + step, .. below e1 (one at least).
template <bool E4M3, int NC>
__device__ __forceinline__ void few_keys(const AttendArgs& a, const Request& rq, int64_t r, int h, const Tiles& tl, const FewRow& fr,
                                         int e0, int step, int e1, FewSums<NC>& st)
{
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int d = a.d, tok = fr.tok, head = fr.head;
    const int64_t per_head = (int64_t)a.page * d;
    const Seen mine = seen_of(a, rq, r, tok);
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

    // the right operand of S^T: channels 64c + 16g .. + 15 of the row
    half8_t qf[NC][2];
    int shift = 0;
    {
        const uint8_t* qp = a.q + 2 * ((int64_t)(rq.start + tok) * a.q_token + head * a.q_head);
        uint4 w[NC][2];
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e = c * 64 + g * 16;
            w[c][0] = w[c][1] = make_uint4(0, 0, 0, 0);
            if (e < d) w[c][0] = *(const uint4*)(qp + 2 * e), w[c][1] = *(const uint4*)(qp + 2 * e + 16);
            if (a.bf16) most = fmaxf(most, fmaxf(abs_most8(w[c][0]), abs_most8(w[c][1])));
        }
        if (a.bf16) shift = row_shift(rows_max(most));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            qf[c][0] = q8(w[c][0], a.bf16, pow2(shift));
            qf[c][1] = q8(w[c][1], a.bf16, pow2(shift));
        }
    }
    const float cap2 = a.softcap * kLog2e;
    const bool large_cap = a.softcap > kSmallCap;
    const float mul = pow2(-shift) * (a.softcap > 0.0f && !large_cap ? a.scale * 2.0f * kLog2e / a.softcap : a.scale * kLog2e);
    const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
    const int pos = rq.pos0 + tok;

    for (int e = e0; e < e1; e += step) {
        // the tile's values, on their way while its scores are formed
        uint4 vw[4 * NC];
        const uint8_t* vp = v_head + pv.id * per_id + pv.in_page * 16 * d;
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) vw[t] = *(const uint4*)(vp + min(t * 16, d - 16) * 16);
        const bool here = pv.here;
        const bool mask = !tile_whole(a, tl, j0) || __any(!here);
        if (!here) sc = make_float2(0.0f, 0.0f);
        const int j0g = j0 + g * 16;
        // scores of keys j0g .. j0g+15 in turn
        float4_t s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<E4M3>(kw[t][c].x, kw[t][c].y), qf[c][0], s[t], 0, 0, 0);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<E4M3>(kw[t][c].z, kw[t][c].w), qf[c][1], s[t], 0, 0, 0);
            }
        }
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
        const float mulk = mul * sc.x;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = s[i >> 2][i & 3] * mulk;
        if (large_cap) {
            const float inv = 1.0f / cap2;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = capped_large(x[i], cap2, inv);
        } else if (a.softcap > 0.0f) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = capped(x[i], cap2);
        }
        if (a.slopes) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] -= slope2 * fabsf((float)(j0g + i - pos));
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
        if (__any(top > st.m + kSlack || vtop > st.vref)) {
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
        sc = sc_next;
    }
    st.l = rows_sum(st.l);
}

// A block a KV head and request, its W waves every W-th tile each, their
// results joined in LDS: for contexts too short to be split.  One sequence of 1024
// tokens, 12 heads of 64: 8.2 us, two tiles a wave in sequence.
template <bool E4M3, int NC, int W>
__global__ __launch_bounds__(64 * W, NC <= 2 ? 2 : 1) void attend_few_kernel(AttendArgs a)
{
    extern __shared__ __align__(16) float lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int d = a.d;
    const int64_t q_heads = (int64_t)a.heads * a.group;
    const int64_t r = blockIdx.x / a.heads;
    const int h = (int)(blockIdx.x % a.heads);
    const Request rq = request_of(a, r);
    if (rq.rows == 0) return;
    const int n_rows = rq.rows * a.group;
    const Tiles tl = few_tiles(a, rq, r);
    FewSums<NC> st;
    if (wave < tl.n) few_keys<E4M3, NC>(a, rq, r, h, tl, few_row(a, rq, h), wave, W, tl.n, st);

    // the waves' parts together: [wave][row] maximum and sum, [wave][row][d] sums
    float* s_m = lds;
    float* s_l = lds + W * kFewRows;
    float* s_acc = lds + 2 * W * kFewRows;
    const int ld = d + 4;
    if (g == 0) s_m[wave * kFewRows + c16] = st.m, s_l[wave * kFewRows + c16] = st.l;
    if (c16 < n_rows) {
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t)
            if (t * 16 < d) *(float4_t*)(s_acc + (wave * kFewRows + c16) * ld + t * 16 + g * 4) = st.acc[t] * (kPart / kTop) * st.vref;
    }
    __syncthreads();
    const int quads = d / 4;
    for (int task = tid; task < n_rows * quads; task += 64 * W) {
        const int rw = task / quads, q4 = task % quads;
        float mm = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < W; ++w) mm = fmaxf(mm, s_m[w * kFewRows + rw]);
        const float m0 = mm == -__builtin_inff() ? 0.0f : mm;
        float ll = 0.0f;
        float4_t o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float k = __builtin_amdgcn_exp2f(s_m[w * kFewRows + rw] - m0);
            ll += k * s_l[w * kFewRows + rw];
            o += k * *(const float4_t*)(s_acc + (w * kFewRows + rw) * ld + 4 * q4);
        }
        const int64_t token = rq.start + rw / a.group;
        const int hq = h * a.group + rw % a.group;
        const float inv = ll == 0.0f ? 0.0f : (1.0f / kPart) / ll;
        *(uint2*)(a.out + 2 * (token * a.o_token + hq * a.o_head + 4 * q4)) =
            make_uint2(f32_to_row2(o[0] * inv, o[1] * inv, a.bf16), f32_to_row2(o[2] * inv, o[3] * inv, a.bf16));
        if (q4 == 0 && a.lse) a.lse[token * q_heads + hq] = ll == 0.0f ? -__builtin_inff() : kLn2 * (mm + __log2f(ll));
    }
}

// Longer contexts.  The tiles of all requests and heads stand in one line,
// request by request and head by head, and every wave takes an equal piece of
// it, so that a batch of any lengths keeps the whole chip busy to the end;
// where a piece ends inside a head's keys its sums go to the workspace and are
// joined by a second kernel.  A piece has two places there, one for the head that
// began before it and one for the head that goes on behind it, so that the
// workspace does not grow with the batch.
// The line's length is only known on the device: each block forms the sum of the
// requests' tiles for itself.  Single tokens, 8 KV heads of 128, groups of four:
// four contexts of 32,768 tokens 59 us (4.6 TB/s; 48 where a part of the codes is
// still in the caches) and the join 5; 64 ragged ones of 1 to 32,768, capped, with a
// bias, 76 us (4.6 TB/s) and 6.
//
// A request's tiles in the line: none without rows, else one at least, so that
// a row that sees no key is written too.  Before each head's tiles stand kBegin
// places that hold none: what beginning a head costs, in tiles.
constexpr int kBegin = 3;
constexpr int kLeastPiece = 2;   // tiles
// Pieces of a head at the most: beyond, the join loses more than the pieces save (one KV head of 128, groups of eight,
// with the bound and without, us: a context of 1,048,576 tokens 85 and 104; two heads, 262,144 tokens 53 and 58).
constexpr int kMostPieces = 512;

__device__ __forceinline__ int line_tiles(const AttendArgs& a, int64_t r)
{
    const Request rq = request_of(a, r);
    return rq.rows == 0 ? 0 : max(1, few_tiles(a, rq, r).n);
}

// A value that is the same in every lane, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

template <bool E4M3, int NC>
__global__ __launch_bounds__(kThreads, NC <= 2 ? 2 : 1) void attend_line_kernel(AttendArgs a)
{
    __shared__ int64_t s_sum[kThreads];
    __shared__ int64_t s_part[kWaves];
    __shared__ int32_t s_most[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int d = a.d;
    const int64_t q_heads = (int64_t)a.heads * a.group;

    // places of the requests before each thread's
    const int64_t per = (a.n_req + kThreads - 1) / kThreads;   // requests of a thread
    int64_t piece, total;
    {
        const int64_t b = min(tid * per, a.n_req), e = min(b + per, a.n_req);
        int64_t sum = 0;
        int most = 0;
        for (int64_t i = b; i < e; ++i) {
            const int t = line_tiles(a, i);
            sum += t ? t + kBegin : 0;
            most = max(most, t);
        }
        int64_t upto = sum;
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
            const int64_t u = __shfl_up(upto, k, 64);
            if (lane >= k) upto += u;
            most = max(most, __shfl_xor(most, k, 64));
        }
        if (lane == 63) s_part[wave] = upto, s_most[wave] = most;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) upto += s_part[w];
            total += s_part[w];
            most = max(most, s_most[w]);
        }
        s_sum[tid] = upto - sum;
        __syncthreads();
        // equal pieces, as long as it takes for no head to be in more than kMostPieces of them
        const int64_t waves = (int64_t)gridDim.x * kWaves;
        total *= a.heads;
        piece = max((total + waves - 1) / waves, (int64_t)(most - 1 + kMostPieces - 2) / (kMostPieces - 1));
        piece = uniform(max(piece, (int64_t)(kBegin + kLeastPiece)));
    }
    // this wave's piece [f, f1) of the line, the request r that it begins in and a head's places before r
    // (neighbouring pieces in different blocks: a short line is spread over all compute units)
    const int64_t number = (int64_t)wave * gridDim.x + blockIdx.x;
    int64_t f = number * piece;
    const int64_t f1 = uniform(min(f + piece, total));
    if (f >= f1) return;
    int lo = 0, hi = kThreads;   // the last thread whose requests begin at or before f
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_sum[mid] * a.heads <= f) lo = mid;
        else hi = mid;
    }
    int64_t r = uniform(lo * per), before = uniform(s_sum[lo]);
    int tiles = line_tiles(a, r), places = tiles ? tiles + kBegin : 0;
    while (f < f1) {
        while (f >= (before + places) * a.heads) {
            before += places;
            tiles = line_tiles(a, ++r);
            places = tiles ? tiles + kBegin : 0;
        }
        const int64_t in_r = f - before * a.heads;
        const int h = (int)(in_r / places);
        const int from = (int)(in_r - (int64_t)h * places);
        const int len = (int)min((int64_t)(places - from), f1 - f);
        const int64_t tile0 = f - from + kBegin;   // where the head's tiles begin in the line
        f += len;
        if (from + len <= kBegin) continue;   // no tile of the head is in the piece
        const int e0 = max(from - kBegin, 0);
        const int split = (int)((tile0 + e0) / piece - tile0 / piece);
        const int n_split = (int)((tile0 + tiles - 1) / piece - tile0 / piece) + 1;

        const Request rq = request_of(a, r);
        const Tiles tl = few_tiles(a, rq, r);
        const int e1 = min(from + len - kBegin, tl.n);
        const FewRow fr = few_row(a, rq, h);
        FewSums<NC> st;
        if (e0 < e1) few_keys<E4M3, NC>(a, rq, r, h, tl, fr, e0, 1, e1, st);
        if (split == 0 && lane == 0) a.pieces[r * a.heads + h] = make_int2(n_split, (int)number);
        if (c16 >= rq.rows * a.group) continue;
        const int64_t token = rq.start + fr.tok;
        if (n_split > 1) {
            const int64_t at = (2 * number + (split == 0)) * a.piece_rows + fr.row;
#pragma unroll
            for (int t = 0; t < 4 * NC; ++t)
                if (t * 16 < d) *(float4_t*)(a.part + at * d + t * 16 + g * 4) = st.acc[t] * (kPart / kTop) * st.vref;
            if (g == 0) a.stat[at] = make_float2(st.m, st.l);
        } else {
            const float inv = st.l == 0.0f ? 0.0f : st.vref * (1.0f / kTop) / st.l;
#pragma unroll
            for (int t = 0; t < 4 * NC; ++t) {
                const float4_t o = st.acc[t] * inv;
                if (t * 16 < d)
                    *(uint2*)(a.out + 2 * (token * a.o_token + fr.head * a.o_head + t * 16 + g * 4)) =
                        make_uint2(f32_to_row2(o[0], o[1], a.bf16), f32_to_row2(o[2], o[3], a.bf16));
            }
            if (g == 0 && a.lse) a.lse[token * q_heads + fr.head] = st.l == 0.0f ? -__builtin_inff() : kLn2 * (st.m + __log2f(st.l));
        }
    }
}

// ------------------------------------------------------------ many rows --

// 32 W rows of one KV head of a request, 32 a wave: what bounds it is the matrix
// products.  A tile's codes are widened to binary16 once, into LDS (two buffers:
// the next tile's codes are on their way from memory meanwhile), and every
// wave takes its left operands from there.  A value channel's keys lie in LDS
// in the order 0-3, 8-11, 4-7, 12-15 of each 16, which is the order in which a
// lane's scores come out of the accumulator.  DP: channels, rounded up.  4096 rows x
// 32 heads of 128 over 32,768 keys 2.0 ms (1.0 PFLOP/s); eight prompts of 500 to
// 2000 rows over 2000 to 8000 keys, capped, 1.30 ms (0.77 PFLOP/s; the vector unit
// busy 57% of the time and the matrix cores 31%, since a wave has a tile's products,
// caps and weights in turn and the waves of a SIMD overlap them only in part).
//
// Blocks go out request by request, the longest context first, so that no long
// one is left for the end: of up to 64 requests, the one with z longer ones.
__device__ __forceinline__ int64_t by_length(const AttendArgs& a, int z)
{
    if (a.n_req == 1 || a.n_req > 64) return z;
    const int n = (int)a.n_req, lane = threadIdx.x & 63;
    const int mine = lane < n ? a.kv_len[lane] : -1;
    int longer = 0;
    for (int j = 0; j < n; ++j) {
        const int other = __builtin_amdgcn_readlane(mine, j);
        longer += (other > mine) | ((other == mine) & (j < lane));
    }
    return __builtin_ctzll(__ballot(lane < n && longer == z));
}

template <int DP, int W>
struct TileLds {
    static constexpr int kRow = DP + 8;       // of a key: channels
    static constexpr int vRow = kTile + 8;    // of a channel: keys
    _Float16 k[2][kTile * kRow];
    _Float16 v[2][DP * vRow];
    int lim[W][6];
};

// PLAIN: neither cap nor bias; the scores then stay as the product gave them up
// to the exponential, which takes their factor, the maximum and the value scale
// in one multiply-add: w = 2^(s c - m + log2 v), v = vs 2^8 / vr, and sum w / v
// is what l wants.  (v is held at 2^-40 from below: values of such a scale are
// zeros, or too small for the sum to notice.)  CAPPED: a small cap and no bias; then
// y = cap (1 - 2 r) with r = 1 / (1 + e^2t), and r stays up to the exponential in
// the same way: the largest score is that of the smallest r, a masked one has r =
// infinity.  FULL: a bias, with or without a small cap.  LARGE: a larger cap, with
// or without a bias; as a branch of FULL it took 3 to 10% of the calls without one
// (registers), and it has no instance for pages of whole tiles.
enum Scores { PLAIN, CAPPED, FULL, LARGE };

// ONE: pages of a multiple of 64 tokens; a tile then lies in one page, with one scale.
template <bool E4M3, int DP, Scores SCORES, bool ONE, int W>
__global__ __launch_bounds__(64 * W, DP <= 64 ? 3 : DP <= 128 ? 2 : 1) void attend_tile_kernel(AttendArgs a)
{
    typedef TileLds<DP, W> Lds;
    constexpr int kThreads = 64 * W, kTileRows = 32 * W;
    extern __shared__ __align__(16) uint8_t raw[];
    Lds& sh = *(Lds*)raw;
    constexpr int G = ONE ? 1 : 4;                                            // parts of a tile that may lie in pages of their own
    constexpr int kChunks = DP / 16;                                          // of a key, 16 codes each
    constexpr int kLoads = (kTile * kChunks + kThreads - 1) / kThreads;       // a thread's loads of each kind
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const int split = (int)(blockIdx.x % a.n_splits);
    const int h = (int)(blockIdx.x / a.n_splits);
    const int64_t r = by_length(a, blockIdx.z);
    const Request rq = request_of(a, r);
    const int n_rows = rq.rows * a.group;
    // the last rows see the most keys: they go first
    const int n_blocks = (n_rows + kTileRows - 1) / kTileRows;
    const int block = n_blocks - 1 - (int)blockIdx.y;
    if (block < 0) return;
    const int d = a.d;
    const int64_t q_heads = (int64_t)a.heads * a.group;

    const int row0 = block * kTileRows + wave * 32;
    const bool used = row0 + c32 < n_rows;
    const int row = min(row0 + c32, n_rows - 1);
    const int tok = row / a.group;
    const int head = h * a.group + row % a.group;
    const Seen mine = seen_of(a, rq, r, tok);
    Tiles tl;
    int wave_lo, wave_hi;   // the keys that some row of the wave sees lie in here
    {
        int v[6] = {mine.lo, -mine.lo, mine.hi, -mine.hi, mine.wlo, -mine.wlo};   // minima, and maxima as minima
#pragma unroll
        for (int k = 1; k < 32; k <<= 1)
#pragma unroll
            for (int i = 0; i < 6; ++i) v[i] = min(v[i], __shfl_xor(v[i], k, 64));
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < 6; ++i) sh.lim[wave][i] = v[i];
        wave_lo = v[0];
        wave_hi = row0 < n_rows ? -v[3] : 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int i = 0; i < 6; ++i) v[i] = min(v[i], sh.lim[w][i]);
        // the same in all lanes: in scalar registers, and with them all that follows from them
#pragma unroll
        for (int i = 0; i < 6; ++i) v[i] = __builtin_amdgcn_readfirstlane(v[i]);
        wave_lo = __builtin_amdgcn_readfirstlane(wave_lo);
        wave_hi = __builtin_amdgcn_readfirstlane(wave_hi);
        tl = tiles_of(a, v[0], -v[1], v[2], -v[3], v[4], -v[5]);
    }
    const int e0 = split * a.split_tiles;
    const int e1 = split == a.n_splits - 1 ? tl.n : min(tl.n, e0 + a.split_tiles);

    float m = -__builtin_inff(), l = 0.0f, vref = kLeast;
    float16_t acc[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] = 0.0f;

    // the right operand of S^T: channels 16s + 8hf .. + 7 of the row
    half8_t qf[kChunks];
    int shift = 0;
    {
        const uint8_t* qp = a.q + 2 * ((int64_t)(rq.start + tok) * a.q_token + head * a.q_head);
        uint4 w[kChunks];
        float most = 0.0f;
#pragma unroll
        for (int s = 0; s < kChunks; ++s) {
            w[s] = make_uint4(0, 0, 0, 0);
            if (s * 16 < d) w[s] = *(const uint4*)(qp + 2 * (s * 16 + hf * 8));
            if (a.bf16) most = fmaxf(most, abs_most8(w[s]));
        }
        if (a.bf16) {
            shift = row_shift(halves_max(most));
        }
        // a negative scale's sign goes into q, so that the factor of a score is not negative
        const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < kChunks; ++s) {
            uint4 u = __builtin_bit_cast(uint4, q8(w[s], a.bf16, pow2(shift)));
            u.x ^= sign, u.y ^= sign, u.z ^= sign, u.w ^= sign;
            qf[s] = __builtin_bit_cast(half8_t, u);
        }
    }
    const float cap2 = a.softcap * kLog2e;
    const float scale = fabsf(a.scale);
    const float mul = pow2(-shift) * (SCORES != LARGE && a.softcap > 0.0f ? scale * 2.0f * kLog2e / a.softcap : scale * kLog2e);
    const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
    const int pos = rq.pos0 + tok;
    const int32_t* table = a.tables + r * a.max_pages;
    const int64_t per_head = (int64_t)a.page * d;

    uint4 kw[kLoads], vw[kLoads];
    // where a thread's loads lie within their part of the tile: channels beyond d come from the last ones
    // (q is zero there, and sums of such channels go nowhere)
    int k_at[kLoads], v_at[kLoads], k_grp[kLoads], v_grp[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        const int q = min(tid + u * kThreads, kTile * kChunks - 1);
        const int key = q / kChunks, kg = q / DP;
        // (a wave's loads are of one group each, but for 96 channels)
        k_grp[u] = DP == 96 ? key >> 4 : __builtin_amdgcn_readfirstlane(key >> 4);
        k_at[u] = (ONE ? key : key & 15) * d + min(q % kChunks * 16, d - 16);
        v_grp[u] = DP == 96 ? kg : __builtin_amdgcn_readfirstlane(kg);
        v_at[u] = ((ONE ? kg * d : 0) + min(q % DP, d - 1)) * 16;
    }
    const uint8_t* k_head = a.k_codes + h * per_head;
    const uint8_t* v_head = a.v_codes + h * per_head;
    const int64_t per_id = a.heads * per_head;
    const float2* scale_head = a.scales + h;
    // The places of a tile's parts are the same for all threads; they are looked up in scalar registers
    // before the barrier that the tile before waits at, so that no load of codes waits for another load.
    Place place[G];
    float2 scales[G];
    bool whole;   // all of the tile's pages are there
    auto look_up = [&](int j0) {
#pragma unroll
        for (int k = 0; k < G; ++k) {
            int grp = (j0 >> 4) + k;
            place[k].here = grp * 16 < rq.kv;
            grp = min(grp, (rq.kv - 1) >> 4);
            const int at = a.per_page_inv ? (int)__umulhi((uint32_t)grp, a.per_page_inv) : grp;
            place[k].in_page = grp - at * (int)a.per_page;
            place[k].id = scalar_load(table + at);
        }
    };
    auto look_up_scales = [&]() {
        whole = true;
#pragma unroll
        for (int k = 0; k < G; ++k) {
            check_place(a, place[k]);
            const uint64_t two = scalar_load((const uint64_t*)(scale_head + (int64_t)place[k].id * a.heads));
            scales[k] = place[k].here ? __builtin_bit_cast(float2, two) : make_float2(0.0f, -1.0f);
            whole = whole && place[k].here;
        }
    };
    auto fetch = [&](int j0) {
        int64_t at[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) at[k] = place[ONE ? 0 : k].id * per_id + place[ONE ? 0 : k].in_page * 16 * d;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            kw[u] = *(const uint4*)(k_head + (ONE ? at[0] : one_of(k_grp[u], at[0], at[1], at[2], at[3])) + k_at[u]);
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            vw[u] = *(const uint4*)(v_head + (ONE ? at[0] : one_of(v_grp[u], at[0], at[1], at[2], at[3])) + v_at[u]);
        if (E4M3 && (!whole || j0 + kTile > rq.kv)) {   // codes after the last key may be anything, a NaN among it
            uint32_t there = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) there |= (uint32_t)place[ONE ? 0 : k].here << k;
#pragma unroll
            for (int u = 0; u < kLoads; ++u)
                vw[u] = first_bytes(vw[u], (there >> v_grp[u]) & 1 ? rq.kv - j0 - 16 * v_grp[u] : 0);
        }
    };
    auto widen = [&](_Float16* ks, _Float16* vs) {   // the codes fetched, into a buffer
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int q = tid + u * kThreads;
            const int key = q / kChunks, c = q % kChunks;
            if (kTile * kChunks % kThreads == 0 || key < kTile) {
                *(half8_t*)(ks + key * Lds::kRow + c * 16) = codes8<E4M3>(kw[u].x, kw[u].y);
                *(half8_t*)(ks + key * Lds::kRow + c * 16 + 8) = codes8<E4M3>(kw[u].z, kw[u].w);
            }
            const int kg = q / DP, ch = q % DP;
            if (kTile * kChunks % kThreads == 0 || kg < 4) {
                *(half8_t*)(vs + ch * Lds::vRow + kg * 16) = codes8<E4M3>(vw[u].x, vw[u].z);
                *(half8_t*)(vs + ch * Lds::vRow + kg * 16 + 8) = codes8<E4M3>(vw[u].y, vw[u].w);
            }
        }
    };
    if (e0 < e1) {
        look_up(tl.tile(e0) * kTile);
        look_up_scales();
        fetch(tl.tile(e0) * kTile);
        widen(sh.k[e0 & 1], sh.v[e0 & 1]);
    }
    for (int e = e0; e < e1; ++e) {
        const int j0 = tl.tile(e) * kTile;
        const _Float16* ks = sh.k[e & 1];
        const _Float16* vs = sh.v[e & 1];
        float2 sn[G];   // the tile's scales
#pragma unroll
        for (int k = 0; k < G; ++k) sn[k] = scales[k];
        const bool all = whole, mask = !all || !tile_whole(a, tl, j0);
        const int jn = tl.tile(min(e + 1, e1 - 1)) * kTile;
        look_up(jn);
        __syncthreads();
        look_up_scales();
        fetch(jn);   // (the last tile once more after itself: it goes nowhere)

        // A wave none of whose rows sees a key of the tile leaves it to the others.  Without and with (us), eight prompts
        // of 500 to 2000 rows over 2000 to 8000 keys: d = 128 1110 and 1057, capped with a prefix 1345 and 1298, with a bias
        // 1289 and 1252; d = 256 1783 and 1666, with a bias 1917 and 1961.  Not at d <= 64, where the widening below then
        // waits for the products: 16 prompts of 1024 rows 82.0 and 83.5, packed documents 64 and 67.
        if (DP <= 64 || (j0 < wave_hi && j0 + kTile > wave_lo)) {
            // x[u*16+i] is the score of key j0 + 32u + 8(i/4) + 4hf + i%4
            float x[32];
            {
                half8_t f[kChunks];
                float16_t s0, s1;
#pragma unroll
                for (int i = 0; i < 16; ++i) s0[i] = s1[i] = 0.0f;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) f[c] = *(const half8_t*)(ks + c32 * Lds::kRow + c * 16 + hf * 8);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    s0 = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[c], qf[c], s0, 0, 0, 0);
                    f[c] = *(const half8_t*)(ks + (32 + c32) * Lds::kRow + c * 16 + hf * 8);
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c) s1 = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[c], qf[c], s1, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = s0[i], x[16 + i] = s1[i];
            }
            // the values of the first two key groups, on their way during the softmax
            half8_t g[DP / 32][2];
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k) g[t][k] = *(const half8_t*)(vs + (t * 32 + c32) * Lds::vRow + k * 16 + hf * 8);
            auto key_of = [&](int i) { return j0 + (i >> 4) * 32 + ((i & 15) >> 2) * 8 + hf * 4 + (i & 3); };
            float c[G];   // factors of the scores
#pragma unroll
            for (int k = 0; k < G; ++k) c[k] = SCORES == PLAIN ? fmaxf(mul * sn[k].x, 0x1p-120f) : mul * sn[k].x;
            if (SCORES == CAPPED) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    x[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * c[ONE ? 0 : i >> 3]));
#pragma unroll
                for (int k = 0; k < G; ++k) c[k] = -2.0f * cap2;
            }
            if (SCORES == FULL || SCORES == LARGE) {
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] *= c[ONE ? 0 : i >> 3];
                if (SCORES == LARGE) {
                    const float inv = 1.0f / cap2;
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = capped_large(x[i], cap2, inv);
                } else if (a.softcap > 0.0f) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = capped(x[i], cap2);
                }
                if (a.slopes) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] -= slope2 * fabsf((float)(key_of(i) - pos));
                }
            }
            constexpr float kHidden = SCORES == CAPPED ? __builtin_inff() : -__builtin_inff();
            if (mask) {
                const uint32_t span = (uint32_t)max(mine.hi - mine.lo, 0);
                const int from = j0 + hf * 4 - mine.lo;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    x[i] = (uint32_t)(from + (i >> 4) * 32 + ((i & 15) >> 2) * 8 + (i & 3)) < span ? x[i] : kHidden;
                if (a.window) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = (key_of(i) >= mine.wlo) | (key_of(i) < a.sinks) ? x[i] : kHidden;
                }
                if (!all) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = sn[ONE ? 0 : i >> 3].y >= 0.0f ? x[i] : kHidden;
                }
            }
            float top = -__builtin_inff(), vtop = -1.0f;
            float tops[G];
#pragma unroll
            for (int k = 0; k < G; ++k) {
                constexpr int n = 32 / G;
                float t = x[n * k];
#pragma unroll
                for (int i = 1; i < n; ++i)
                    t = SCORES == CAPPED ? __builtin_elementwise_minimum(t, x[n * k + i]) : __builtin_elementwise_maximum(t, x[n * k + i]);
                top = __builtin_elementwise_maximum(top, SCORES == PLAIN ? t * c[k] : SCORES == CAPPED ? __builtin_fmaf(t, c[k], cap2) : t);
                vtop = fmaxf(vtop, sn[k].y);
                tops[k] = t;
            }
            top = halves_max(top);
            if (mask) {   // only of parts of which the row sees a key
                vtop = -1.0f;
#pragma unroll
                for (int k = 0; k < G; ++k) vtop = fmaxf(vtop, tops[k] != kHidden ? sn[k].y : -1.0f);
                vtop = halves_max(vtop);
            }
            if (__any(top > m + kSlack || vtop > vref)) {
                const float mnew = fmaxf(m, top), vnew = fmaxf(vref, vtop);
                const float shrink = mnew == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - mnew);
                l *= shrink;
                const float f = shrink * (vref / vnew);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) acc[t] *= f;
                m = mnew;
                vref = vnew;
            }
            const float m0 = m == -__builtin_inff() ? 0.0f : m;
            const float vmul = kTop / vref;
            float vb[G], vinv[G];
#pragma unroll
            for (int k = 0; k < G; ++k) {
                const float v = __builtin_amdgcn_fmed3f(sn[k].y * vmul, 0x1p-40f, kTop);   // (more only where nothing is seen)
                vb[k] = __builtin_amdgcn_logf(v) - m0 + (SCORES == CAPPED ? cap2 : 0.0f);
                vinv[k] = __builtin_amdgcn_rcpf(v);
            }
            auto weights = [&](int k) {   // of keys 16k .. 16k+15, this lane's half of them
                const int part = ONE ? 0 : k;
                float sum = 0.0f;
                half8_t p;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float w = __builtin_amdgcn_exp2f(SCORES == PLAIN || SCORES == CAPPED ? __builtin_fmaf(x[8 * k + i], c[part], vb[part]) : x[8 * k + i] + vb[part]);
                    sum += w;
                    p[i] = (_Float16)w;
                }
                l = __builtin_fmaf(sum, vinv[part], l);
                return p;
            };
            const half8_t p0 = weights(0), p1 = weights(1);
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) {
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g[t][0], p0, acc[t], 0, 0, 0);
                g[t][0] = *(const half8_t*)(vs + (t * 32 + c32) * Lds::vRow + 2 * 16 + hf * 8);
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g[t][1], p1, acc[t], 0, 0, 0);
                g[t][1] = *(const half8_t*)(vs + (t * 32 + c32) * Lds::vRow + 3 * 16 + hf * 8);
            }
            const half8_t p2 = weights(2), p3 = weights(3);
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) {
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g[t][0], p2, acc[t], 0, 0, 0);
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g[t][1], p3, acc[t], 0, 0, 0);
            }
        }
        widen(sh.k[(e + 1) & 1], sh.v[(e + 1) & 1]);
    }
    l = halves_sum(l);
    if (!used) return;
    const int64_t token = rq.start + tok;
    if (a.n_splits > 1) {
        const int64_t at = (token * q_heads + head) * a.n_splits + split;
        if (hf == 0) a.stat[at] = make_float2(m, l);
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ch = t * 32 + i * 8 + hf * 4;
                if (ch < d)
                    *(float4_t*)(a.part + at * d + ch) =
                        float4_t{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]} * (kPart / kTop) * vref;
            }
        return;
    }
    const float inv = l == 0.0f ? 0.0f : vref * (1.0f / kTop) / l;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ch = t * 32 + i * 8 + hf * 4;
            if (ch < d)
                *(uint2*)(a.out + 2 * (token * a.o_token + head * a.o_head + ch)) =
                    make_uint2(f32_to_row2(acc[t][4 * i] * inv, acc[t][4 * i + 1] * inv, a.bf16),
                               f32_to_row2(acc[t][4 * i + 2] * inv, acc[t][4 * i + 3] * inv, a.bf16));
        }
    if (hf == 0 && a.lse) a.lse[token * q_heads + head] = l == 0.0f ? -__builtin_inff() : kLn2 * (m + __log2f(l));
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
    if (item >= a.n_req * a.max_new * q_heads) return;
    const int64_t r = item / (a.max_new * q_heads);
    const int64_t i = item / q_heads % a.max_new;
    const int64_t hq = item % q_heads;
    const Request rq = request_of(a, r);
    if (i >= rq.rows) return;
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

// ------------------------------------------------------------------ host --

struct Shape {
    bool few;
    int tile_waves;       // of the kernel for many rows, 32 rows each,
    int64_t row_blocks;   // and its blocks of a request and KV head
    int64_t blocks;       // of the kernel for few rows,
    int few_waves;        // and their waves
    int n_splits, split_tiles;   // (few rows: 1, or more than 1 for the line)
    bool join_blocks;     // a block joins a row's splits, not a wave
};

constexpr int64_t kFewBlocks = 512;   // two on each compute unit

// The kernel for few rows where a KV head's rows fit one of its blocks.  Its
// keys are split where the heads alone leave compute units idle or the longest
// request may hold up the rest; how the tiles are dealt is settled on the device.
// The other kernel's keys are split so
// that about four hundred blocks are there, with four tiles for a block at the
// least.
Shape shape_of(const fkv_page_desc* p, const fkv_attend_desc* t)
{
    Shape s = {};
    const int64_t group = t->q_heads / p->heads;
    const int64_t rows = t->max_new * group;
    s.few = rows <= kFewRows;
    // Eight waves share a tile's widening, four make finer blocks, two of which fill a compute unit with
    // phases of their own.  Measured with 4 and 8 (us), 8 KV heads of 128: a 4096-token chunk over 32,768 keys, groups
    // of four, 2207 and 2036; one prompt of 4096 169 and 165; eight of 500 to 2000 rows over 2000 to 8000 keys 1088 and
    // 1075, with a bias 1302 and 1281, capped 1278 and 1308.  Fewer rows: 40 x 4 heads over 8192 keys 19.6 and 20.9,
    // 16 prompts of 2048 with one query head a KV head 216 and 255.  Uneven: 16 of 100 to 4096 rows 264 and 275.
    // d = 64, 16,384 rows 589 and 700.
    const bool even = 4 * t->n_tokens >= 3 * t->n_req * t->max_new;   // the requests' rows are about as many
    s.tile_waves = p->d > 64 && p->d <= 128 && rows >= 4096 && even ? 8 : 4;
    s.row_blocks = s.few ? 1 : (rows + 32 * s.tile_waves - 1) / (32 * s.tile_waves);
    const int64_t kv = min(t->max_kv, t->max_pages * p->page);
    int64_t tiles = (kv + kTile - 1) / kTile;
    if (t->window)   // no more than the window's and the sinks' tiles are seen
        tiles = min(tiles, ((int64_t)t->window + t->max_new + kTile - 1) / kTile + 1 + ((int64_t)t->sinks + kTile - 1) / kTile);
    tiles = max(tiles, (int64_t)1);
    const int64_t heads = max((int64_t)1, t->n_req * p->heads);
    if (s.few) {
        s.few_waves = kWaves;
        if (tiles <= 16) {
            s.n_splits = 1;
            s.blocks = heads;
            if (p->d <= 128 && heads <= kFewBlocks / 2 && tiles > kWaves) s.few_waves = 8;
        } else {
            s.n_splits = 2;
            s.blocks = kFewBlocks;
            s.join_blocks = heads <= kFewBlocks && tiles >= kManySplits * kLeastPiece;
        }
        return s;
    }
    // (the two may be any numbers: their product only where it is small)
    const int64_t want = heads >= 400 || s.row_blocks >= 400 ? 1 : (400 + heads * s.row_blocks - 1) / (heads * s.row_blocks);
    const int64_t most = max((int64_t)1, tiles / kWaves);
    const int64_t n = max((int64_t)1, min(want, most));
    s.split_tiles = (int)((tiles + n - 1) / n);
    s.n_splits = (int)((tiles + s.split_tiles - 1) / s.split_tiles);
    s.join_blocks = s.n_splits >= kManySplits;
    return s;
}

bool attend_ok(const fkv_page_desc* p, const fkv_attend_desc* t)
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

// The workspace: sums, then maxima and sums of weights, then the heads' pieces of the line.
struct Workspace {
    size_t stat, pieces, bytes;
};

Workspace workspace_of(const fkv_page_desc* p, const fkv_attend_desc* t, const Shape& s)
{
    if (s.n_splits == 1) return Workspace{0, 0, 0};
    const size_t rows = s.few ? (size_t)s.blocks * kWaves * 2 * (t->max_new * (t->q_heads / p->heads))
                              : (size_t)t->n_tokens * t->q_heads * s.n_splits;
    Workspace w;
    w.stat = rows * p->d * sizeof(float);
    w.pieces = w.stat + rows * sizeof(float2);
    w.bytes = w.pieces + (s.few ? (size_t)t->n_req * p->heads * sizeof(int2) : 0);
    return w;
}

}  // namespace
}  // namespace fkv

using namespace fkv;

extern "C" size_t fkv_page_attend_workspace(const fkv_page_desc* desc, const fkv_attend_desc* attend)
{
    if (!attend_ok(desc, attend)) return 0;
    return workspace_of(desc, attend, shape_of(desc, attend)).bytes;
}

extern "C" int fkv_page_attend(const fkv_page_desc* desc, const fkv_attend_desc* attend, const uint8_t* k_codes,
                               const uint8_t* v_codes, const float* scales, const void* q, const int32_t* tables,
                               const int32_t* kv_len, const int32_t* q_start, const float* slopes,
                               const int32_t* prefix, const int32_t* first, void* out, float* lse, void* workspace,
                               size_t workspace_bytes, void* stream)
{
    if (!attend_ok(desc, attend)) return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8))
        return FKV_ERR_INVALID_ARG;
    if (attend->n_req == 0 || attend->n_tokens == 0) return FKV_OK;
    if (!q || !out || !tables || !kv_len || !q_start || !aligned(q, 16) || !aligned(out, 16) || !aligned(tables, 4) ||
        !aligned(kv_len, 4) || !aligned(q_start, 4) || !aligned(slopes, 4) || !aligned(prefix, 4) ||
        !aligned(first, 4) || !aligned(lse, 4) || !aligned(workspace, 16))
        return FKV_ERR_INVALID_ARG;
    const Shape s = shape_of(desc, attend);
    const Workspace ws = workspace_of(desc, attend, s);
    if (ws.bytes && (!workspace || workspace_bytes < ws.bytes)) return FKV_ERR_SCRATCH_TOO_SMALL;
    AttendArgs a = {};
    a.k_codes = k_codes, a.v_codes = v_codes, a.scales = (const float2*)scales;
    a.q = (const uint8_t*)q, a.out = (uint8_t*)out, a.lse = lse;
    a.tables = tables, a.kv_len = kv_len, a.q_start = q_start;
    a.slopes = slopes, a.prefix = prefix, a.first = first;
    a.part = (float*)workspace;
    a.stat = (float2*)((uint8_t*)workspace + ws.stat);
    a.pieces = ws.bytes && s.few ? (int2*)((uint8_t*)workspace + ws.pieces) : nullptr;
    a.n_req = attend->n_req, a.n_tokens = attend->n_tokens, a.max_new = attend->max_new, a.max_kv = attend->max_kv;
    a.max_pages = attend->max_pages, a.n_pages = desc->n_pages;
    a.q_token = attend->q_stride_token, a.q_head = attend->q_stride_head;
    a.o_token = attend->o_stride_token, a.o_head = attend->o_stride_head;
    a.page = desc->page, a.heads = desc->heads, a.group = attend->q_heads / desc->heads, a.d = desc->d;
    a.window = attend->window, a.sinks = attend->sinks;
    a.bf16 = attend->type, a.causal = attend->causal;
    a.n_splits = s.n_splits, a.split_tiles = s.split_tiles;
    a.piece_rows = s.few ? (int32_t)(attend->max_new * a.group) : 0;
    a.per_page = (uint32_t)(desc->page / 16);
    a.per_page_inv = a.per_page == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + a.per_page - 1) / a.per_page);
    a.scale = attend->scale, a.softcap = attend->softcap;
    const hipStream_t st = (hipStream_t)stream;
    const bool e4m3 = desc->format == FKV_PAGE_E4M3;
    // what a launch cannot hold is refused before the first
    const int64_t items = s.n_splits > 1 ? a.n_req * a.max_new * a.heads * a.group : 0;   // rows to be joined
    const int64_t joins = s.join_blocks ? items : (items + kWaves - 1) / kWaves;
    if (joins > 0x7fffff00 || s.blocks > 0x7fffff00) return FKV_ERR_UNSUPPORTED;
    if (s.few) {
        auto go = [&](auto kern, int w) {
            const size_t shm = (2 * w * kFewRows + (size_t)w * kFewRows * (a.d + 4)) * sizeof(float);
            hipLaunchKernelGGL(kern, dim3((unsigned)s.blocks), dim3(64 * w), shm, st, a);
        };
        auto of_width = [&](auto nc) {
            constexpr int NC = decltype(nc)::value;
            if (s.n_splits > 1) {
                auto kern = e4m3 ? attend_line_kernel<true, NC> : attend_line_kernel<false, NC>;
                hipLaunchKernelGGL(kern, dim3((unsigned)s.blocks), dim3(kThreads), 0, st, a);
                return;
            }
            if constexpr (NC <= 2) {
                if (s.few_waves == 8) {
                    e4m3 ? go(attend_few_kernel<true, NC, 8>, 8) : go(attend_few_kernel<false, NC, 8>, 8);
                    return;
                }
            }
            e4m3 ? go(attend_few_kernel<true, NC, 4>, 4) : go(attend_few_kernel<false, NC, 4>, 4);
        };
        if (a.d <= 64) of_width(std::integral_constant<int, 1>{});
        else if (a.d <= 128) of_width(std::integral_constant<int, 2>{});
        else of_width(std::integral_constant<int, 4>{});
    } else {
        if (s.row_blocks > 65535 || a.n_req > 65535 || (int64_t)a.heads * a.n_splits > 0x7fffff00) return FKV_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)(a.heads * a.n_splits), (unsigned)s.row_blocks, (unsigned)a.n_req);
        // (a launch may take all of a block's 160 KB of LDS; the widest tiles take 141)
        auto go = [&](auto kern, size_t shm, int w) { hipLaunchKernelGGL(kern, grid, dim3(64 * w), shm, st, a); };
        auto of_waves = [&](auto dp, auto waves) {
            constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
            constexpr size_t shm = sizeof(TileLds<DP, W>);
            auto of_scores = [&](auto scores) {
                constexpr Scores S = decltype(scores)::value;
                if constexpr (S != LARGE) {
                    if (a.page % kTile == 0) {
                        e4m3 ? go(attend_tile_kernel<true, DP, S, true, W>, shm, W) : go(attend_tile_kernel<false, DP, S, true, W>, shm, W);
                        return;
                    }
                }
                e4m3 ? go(attend_tile_kernel<true, DP, S, false, W>, shm, W) : go(attend_tile_kernel<false, DP, S, false, W>, shm, W);
            };
            if (a.softcap > kSmallCap) of_scores(std::integral_constant<Scores, LARGE>{});
            else if (a.slopes) of_scores(std::integral_constant<Scores, FULL>{});
            else if (a.softcap > 0.0f) of_scores(std::integral_constant<Scores, CAPPED>{});
            else of_scores(std::integral_constant<Scores, PLAIN>{});
        };
        auto of_width = [&](auto dp) {
            if constexpr (decltype(dp)::value == 96 || decltype(dp)::value == 128) {
                if (s.tile_waves == 8) return of_waves(dp, std::integral_constant<int, 8>{});
            }
            of_waves(dp, std::integral_constant<int, 4>{});
        };
        if (a.d <= 64) of_width(std::integral_constant<int, 64>{});
        else if (a.d <= 96) of_width(std::integral_constant<int, 96>{});
        else if (a.d <= 128) of_width(std::integral_constant<int, 128>{});
        else of_width(std::integral_constant<int, 256>{});
    }
    if (a.n_splits > 1)
        hipLaunchKernelGGL(s.join_blocks ? attend_join_kernel<kWaves> : attend_join_kernel<1>, dim3((unsigned)joins), dim3(kThreads), 0, st, a);
    return launch_status();
}
