// page_select_kernels.hip -- attention to a few pages of a long context, for
// gfx950: a bound on the scores of each page's keys, the pages with the largest
// bounds for each query token and KV head, and attention over lists of pages.
//
// A page's box holds the smallest and largest code of every key channel, lo and hi,
// so that no key of the page has a product with q above
//     sum_c max(q_c lo_c, q_c hi_c) = sum_c q+_c hi_c + q-_c lo_c,
// with q+ and q- the positive and negative parts of q: a matrix product of twice the
// keys' width.  It is formed of whole numbers, q being rounded to 8 bits with a power
// of two for each row, so that it is exact in any order: which pages are selected does
// not depend on how the work is dealt out.
#include "page_attend_device.h"

#include <algorithm>

namespace fkv {
namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));

struct SelectArgs : AttendArgs {
    const uint8_t* boxes;
    int32_t* scores;    // [token][KV head][score_stride], as ordered() gives them
    int32_t* selected;  // [token][KV head][n_select]
    int64_t score_stride;
    int64_t row_groups;   // of the scoring kernel: row tiles of a request, R a block
    int64_t searched_groups;   // or of all requests, which the kernel looks up (0: row_groups a request)
    int32_t n_select, keep_first, keep_last;
    int32_t tile_chunks;  // and its blocks along the pages, of wave_tiles tiles of 16 pages a wave
    int32_t wave_tiles;
    int32_t lanes_log;    // a token's rows of a tile: a power of two of them
};

__device__ __forceinline__ int pages_of(const AttendArgs& a, int tokens)   // tokens >= 0
{
    const uint32_t groups = (uint32_t)((int64_t)tokens + 15) >> 4;
    if (groups == 0) return 0;
    return (int)(a.per_page_inv ? __umulhi(groups - 1, a.per_page_inv) : groups - 1) + 1;
}

// The pages that token i of a request may select from.
__device__ __forceinline__ int pages_seen(const AttendArgs& a, const Request& rq, int i)
{
    const int end = a.causal ? min(rq.pos0 + i + 1, rq.kv) : rq.kv;
    return pages_of(a, max(end, 0));
}

// The request and row of a launch's place for a token; r -1: of none, i -1: to be told from the request's first row.
struct TokenPlace {
    int64_t r;
    int i;
};

__device__ __forceinline__ TokenPlace token_place(const AttendArgs& a, uint32_t place)
{
    if (a.searched) return TokenPlace{request_at(a, place, 1), -1};
    const uint32_t r = place / (uint32_t)a.max_new;
    return TokenPlace{r, (int)(place - r * (uint32_t)a.max_new)};
}

// ---------------------------------------------------------------- scores --

// Four codes of a box as 8-bit whole numbers: int8 codes as they are, 8-bit floats
// in units of 4, rounded away from the box's inside (HIGH: up).
template <bool E4M3, bool HIGH>
__device__ __forceinline__ uint32_t whole4(uint32_t w)
{
    if (!E4M3) return w;
    float f[4];
    codes_to_f32<true>(w, f);
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = (uint32_t)(int)(HIGH ? ceilf(f[e] * 0.25f) : floorf(f[e] * 0.25f));
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

template <bool E4M3, bool HIGH>
__device__ __forceinline__ int4_t whole16(uint4 w)
{
    return int4_t{(int)whole4<E4M3, HIGH>(w.x), (int)whole4<E4M3, HIGH>(w.y), (int)whole4<E4M3, HIGH>(w.z), (int)whole4<E4M3, HIGH>(w.w)};
}

// A score as a whole number, in the order of the scores; one that is a NaN as -infinity.
__device__ __forceinline__ int ordered(float x)
{
    const int u = __builtin_bit_cast(int, fmaxf(x, -__builtin_inff()));   // (the larger of a NaN and another number is the other)
    return u ^ (int)((uint32_t)(u >> 31) >> 1);
}

// The largest of the lanes that share all bits of their number but the lowest `log` (up
// to four), of N values at once.
template <int N>
__device__ __forceinline__ void lanes_max(int (&v)[N], int log)
{
    auto with = [&](auto ctrl) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = max(v[i], __builtin_amdgcn_update_dpp(v[i], v[i], decltype(ctrl)::value, 0xf, 0xf, false));
    };
    if (log > 0) with(std::integral_constant<int, 0xb1>{});    // with the neighbour,
    if (log > 1) with(std::integral_constant<int, 0x4e>{});    // the other pair of four,
    if (log > 2) with(std::integral_constant<int, 0x141>{});   // the other four of eight,
    if (log > 3) with(std::integral_constant<int, 0x140>{});   // the other eight
}

// Rows of q as whole numbers, a tile of 16 -- a few tokens' heads of one KV head, or
// up to 16 of one token's -- in LDS: positive and negative parts, and 2^-e.  A wave
// rounds four rows at a time, 16 lanes a row and 8 channels a lane.
template <int NC, int R>
struct RowsLds {
    static constexpr int kDepth = NC * 64, kRow = 2 * kDepth + 16;   // bytes (16 more: rows begin in banks of their own)
    uint8_t part[R * 16 * kRow];
    float mul[R * 16];
};

template <int NC>
__device__ __forceinline__ void round_row(const SelectArgs& a, const uint8_t* qp, uint8_t* to, float* mul_to)
{
    constexpr int kParts = NC <= 2 ? 1 : 2;   // of 128 channels
    const int c16 = threadIdx.x & 15;
    uint4 w[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        const int ch = k * 128 + c16 * 8;
        w[k] = make_uint4(0, 0, 0, 0);
        if (ch < a.d) w[k] = *(const uint4*)(qp + 2 * ch);
    }
    auto element = [&](int k, int e) {
        const uint32_t pair[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        return row_to_f32(pair[e >> 1], e & 1, a.bf16);
    };
    // the row's largest; `strange` is a NaN once an element is none or infinite
    float most = 0.0f, strange = 0.0f;
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            most = fmaxf(most, fabsf(element(k, e)));
            strange = __builtin_fmaf(element(k, e), 0.0f, strange);
        }
    const bool special = __any(strange != strange);
    if (special) {
        most = 0.0f;
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(element(k, e)) < __builtin_inff() ? fabsf(element(k, e)) : 0.0f);
    }
    int all[1] = {__builtin_bit_cast(int, most)};   // (of numbers that are not negative the bits are in their order)
    lanes_max(all, 4);
    most = __builtin_bit_cast(float, all[0]);
    const int ex = (int)(__float_as_uint(most) >> 23);
    const int e2 = ex == 0 ? 0 : min(133 - ex, 126);
    const float mul = pow2(e2), most_whole = 127.0f * pow2(-e2);
    if (c16 == 0) *mul_to = pow2(-e2);
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        const int ch = k * 128 + c16 * 8;
        uint32_t plus[2], minus[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t u[4];   // x * mul + 1.5 2^23 has the whole number, rounded to nearest with ties to even, in its low bits
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = element(k, 4 * q + e);
                if (special) x = x == x ? x : 0.0f;
                u[e] = __float_as_uint(__builtin_fmaf(__builtin_amdgcn_fmed3f(x, -most_whole, most_whole), mul, 12582912.0f));
            }
            const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u);
            const uint32_t four = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
            const uint32_t negative = ((four >> 7) & 0x01010101u) * 0xffu;   // the bytes of negative numbers
            plus[q] = four & ~negative;
            minus[q] = four & negative;
        }
        if (ch < NC * 64) {   // (zeros beyond d)
            *(uint2*)(to + ch) = make_uint2(plus[0], plus[1]);
            *(uint2*)(to + NC * 64 + ch) = make_uint2(minus[0], minus[1]);
        }
    }
}

// The WAVES waves of a block form the scores of R tiles of 16 rows of one KV head of a
// request, from token tok0 on, this wave of n_tiles tiles of 16 pages: `first`, first +
// step, ..  The left operand takes a page's box as one of its rows, so that lane 16g + c
// ends up with row c's sums of pages 4g .. 4g+3.  Of KV heads of more than 16 rows (WIDE) a
// block has one token, and R tiles of its rows at a time.  put(token, page, scores, c0) gets
// four pages' scores; c0: the heads are not the first ones.
template <bool E4M3, int NC, int R, bool WIDE, int WAVES, typename Put>
__device__ __forceinline__ void score_block(const SelectArgs& a, const Request& rq, int64_t r, int h, int tok0, int most_seen, int first,
                                            int step, int n_tiles, RowsLds<NC, R>& sh, Put put)
{
    typedef RowsLds<NC, R> Lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int chunks = WIDE ? (a.group + 15) >> 4 : 1;   // of a token's heads, 16 a tile
    const int per_tile = 16 >> a.lanes_log;              // tokens of a tile
    const int32_t* table = a.tables + r * a.max_pages;
    int kc[NC];   // channels beyond d are taken from the last ones: q is zero there
#pragma unroll
    for (int c = 0; c < NC; ++c) kc[c] = min(c * 64 + g * 16, a.d - 16);
    struct Pages {
        uint4 lo[NC], hi[NC];
        float scale;   // of page c16; a NaN where there is none
    };
    auto id_of = [&](int k) { return table[min((first + k * step) * 16 + c16, most_seen - 1)]; };
    auto load = [&](int id) {
        Pages p;
        const bool here = (uint32_t)id < (uint64_t)a.n_pages;
        const int64_t at = (here ? id : 0) * (int64_t)a.heads + h;
        p.scale = here ? a.scales[at].x : __builtin_nanf("");
        const uint8_t* box = a.boxes + at * 2 * a.d;
#pragma unroll
        for (int c = 0; c < NC; ++c) p.lo[c] = *(const uint4*)(box + kc[c]), p.hi[c] = *(const uint4*)(box + a.d + kc[c]);
        return p;
    };
    const int lanes = 1 << a.lanes_log;
    for (int c0 = 0; c0 < chunks; c0 += R) {
        // (tiles of no token are left out)
        const int row_tiles = WIDE ? min(R, chunks - c0) : min(R, (rq.rows - tok0 + per_tile - 1) / per_tile);
        int id1 = id_of(min(1, max(n_tiles - 1, 0)));
        Pages next = load(id_of(0));   // (of a wave without a tile: the last page, for nothing)
        if (c0) __syncthreads();
        // rows 4 (wave + WAVES k) + g of the block's tiles
        for (int k = wave * 4; k < row_tiles * 16; k += WAVES * 4) {
            const int row = k + g, t = row >> 4, in_tile = row & 15;
            const int tok = min(WIDE ? tok0 : tok0 + t * per_tile + (in_tile >> a.lanes_log), rq.rows - 1);
            const int in_group = min(WIDE ? (c0 + t) * 16 + in_tile : in_tile & (lanes - 1), a.group - 1);
            round_row<NC>(a, a.q + 2 * ((int64_t)(rq.start + tok) * a.q_token + (h * a.group + in_group) * a.q_head),
                          sh.part + row * Lds::kRow, sh.mul + row);
        }
        __syncthreads();
        for (int k = 0; k < n_tiles; ++k) {
            if (WAVES > kWaves) asm volatile("" ::: "memory");   // (the rows' operands stay in LDS: a block of many waves has no registers for them)
            const Pages now = next;
            if (k + 1 < n_tiles) {
                next = load(id1);
                id1 = id_of(min(k + 2, n_tiles - 1));
            }
            int4_t lo[NC], hi[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) lo[c] = whole16<E4M3, false>(now.lo[c]), hi[c] = whole16<E4M3, true>(now.hi[c]);
            float scale[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) scale[i] = __shfl(now.scale, 4 * g + i, 64);
            int x[4];
#pragma unroll
            for (int t = 0; t < R; ++t) {
                if (t && t >= row_tiles) break;
                const uint8_t* rows = sh.part + (t * 16 + c16) * Lds::kRow + g * 16;
                int4_t sum = {0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi[c], *(const int4_t*)(rows + c * 64), sum, 0, 0, 0);
                    sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(lo[c], *(const int4_t*)(rows + Lds::kDepth + c * 64), sum, 0, 0, 0);
                }
                const float mul = sh.mul[t * 16 + c16];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int y = ordered(((float)sum[i] * scale[i]) * mul);
                    x[i] = WIDE && t ? max(x[i], y) : y;
                }
                if (WIDE && t + 1 < row_tiles) continue;
                lanes_max(x, a.lanes_log);
                const int tok = WIDE ? tok0 : tok0 + t * per_tile + (c16 >> a.lanes_log);
                if ((c16 & (lanes - 1)) == 0 && tok < rq.rows) put(tok, (first + k * step) * 16 + g * 4, int4_t{x[0], x[1], x[2], x[3]}, WIDE && c0);
            }
        }
    }
}

// Many rows or many pages: the scores go to the workspace (16 contexts of 2048 pages, 8 heads
// of 128: 67 MB of boxes, 19.5 us, 3.4 TB/s; a chunk's rows over 512 pages: 57 us, the vector
// unit 76% busy, that turns sums to scores and joins the heads, the matrix cores 13%).  A block R row tiles, a wave of it
// a quarter of the block's page tiles.
template <bool E4M3, int NC, int R, bool WIDE>
__global__ __launch_bounds__(kThreads, R == 1 || NC == 1 ? 4 : NC == 2 ? 3 : 2) void page_score_kernel(SelectArgs a)
{
    __shared__ __align__(16) RowsLds<NC, R> sh;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t b = blockIdx.x;
    const int h = (int)(b % (uint32_t)a.heads);
    b /= (uint32_t)a.heads;
    const int chunk = (int)(b % (uint32_t)a.tile_chunks);
    b /= (uint32_t)a.tile_chunks;
    const int tokens = WIDE ? 1 : R * (16 >> a.lanes_log);   // of the block
    int64_t r;
    int rg;
    if (a.searched_groups) {
        r = request_at(a, b, tokens);
        if (r < 0) return;
        rg = (int)(b - first_place(a, r, tokens));
    } else {
        r = b / (uint32_t)a.row_groups;
        rg = (int)(b - (uint32_t)r * (uint32_t)a.row_groups);
    }
    const Request rq = request_of(a, r);
    if (rg < 0 || (int64_t)rg * tokens >= rq.rows) return;   // (negative: of starts out of order)
    const int tok0 = rg * tokens;
    const int most_seen = pages_seen(a, rq, min(tok0 + tokens, rq.rows) - 1);   // (later tokens see no fewer)
    if (most_seen <= a.n_select) return;   // every page of theirs is selected
    const int tiles = (most_seen + 15) >> 4;
    const int first_of_block = chunk * a.wave_tiles * kWaves;
    if (first_of_block >= tiles) return;
    const int first = first_of_block + wave * a.wave_tiles;
    score_block<E4M3, NC, R, WIDE, kWaves>(a, rq, r, h, tok0, most_seen, first, 1, max(min(a.wave_tiles, tiles - first), 0), sh,
                                           [&](int tok, int page, int4_t x, bool again) {
        int4_t* to = (int4_t*)(a.scores + ((rq.start + tok) * (int64_t)a.heads + h) * a.score_stride + page);
        if (again) {   // with the heads before
            const int4_t before = *to;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = max(x[i], before[i]);
        }
        *to = x;
    });
}

// ------------------------------------------------------------- selection --

// The scores' order without a sign, none of them 0.
__device__ __forceinline__ uint32_t key_of_score(int x)
{
    return (uint32_t)(x == -1 ? 0 : x) ^ 0x80000000u;   // (-0, in order -1, is 0)
}

// A row of the lists: token, KV head, and how many pages the token sees.
struct SelectRow {
    int64_t at;   // token * heads + h
    int seen;
    bool any;
};

__device__ __forceinline__ SelectRow select_row(const SelectArgs& a, uint32_t item)   // (below 2^31)
{
    SelectRow s = {0, 0, false};
    if (item >= (uint32_t)((a.searched ? a.searched : a.n_req * a.max_new) * a.heads)) return s;
    const uint32_t ri = item / (uint32_t)a.heads;
    const int h = (int)(item - ri * (uint32_t)a.heads);
    const TokenPlace at = token_place(a, ri);
    if (at.r < 0) return s;
    const Request rq = request_of(a, at.r);
    const int i = at.i < 0 ? (int)ri - rq.start : at.i;
    if ((uint32_t)i >= (uint32_t)rq.rows) return s;   // (negative: of starts out of order)
    s.at = (rq.start + i) * (int64_t)a.heads + h;
    s.seen = pages_seen(a, rq, i);
    s.any = true;
    return s;
}

// The W waves of a row write its list, its scores in registers: page 64 (N wave + n) +
// lane in key[n].  The smallest score selected is found bit by bit from the first that the
// scores differ in; each step counts those above by ballots, and the search ends when the
// count fits.
template <int W>
struct PickLds {
    uint32_t top[W], low[W];
    int count[2][W], same[W];
};

template <int N, int W>
__device__ __forceinline__ void pick_pages(const SelectArgs& a, int seen, const int32_t* scores, int32_t* out, int wave, PickLds<W>& sh)
{
    const int lane = threadIdx.x & 63, thread = wave * 64 + lane;
    if (seen <= a.n_select) {
        for (int j = thread; j < a.n_select; j += 64 * W) out[j] = j < seen ? j : -1;
        return;
    }
    // (more pages than are selected: those always kept are apart from each other)
    const int from = a.keep_first, to = seen - a.keep_last, want = a.n_select - a.keep_first - a.keep_last;
    const int page0 = wave * N * 64 + lane;
    uint32_t key[N];
    int score[N];
#pragma unroll
    for (int n = 0; n < N; ++n) score[n] = scores[min(page0 + 64 * n, seen - 1)];   // (without a condition: all on their way at once)
#pragma unroll
    for (int n = 0; n < N; ++n) key[n] = page0 + 64 * n >= from && page0 + 64 * n < to ? key_of_score(score[n]) : 0u;
    uint32_t top = 0, low = 0xffffffffu;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        top = max(top, key[n]);
        low = min(low, key[n] ? key[n] : 0xffffffffu);
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        top = max(top, (uint32_t)__shfl_xor((int)top, k, 64));
        low = min(low, (uint32_t)__shfl_xor((int)low, k, 64));
    }
    if (W > 1) {
        if (lane == 0) sh.top[wave] = top, sh.low[wave] = low;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) top = max(top, sh.top[w]), low = min(low, sh.low[w]);
    }
    top = __builtin_amdgcn_readfirstlane(top);
    low = __builtin_amdgcn_readfirstlane(low);
    int turn = 0;
    auto over_row = [&](int c) {   // a count of the wave's, over the row's waves
        if (W == 1) return c;
        turn ^= 1;
        if (lane == 0) sh.count[turn][wave] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += sh.count[turn][w];
        return (int)__builtin_amdgcn_readfirstlane(c);
    };
    auto count = [&](uint32_t least) {
        int c = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) c += __builtin_popcountll(__ballot(key[n] >= least));
        return c;
    };
    // the largest t of which `want` scores or more are not below; of those equal to it the first `ties` are taken
    uint32_t t = 0xffffffffu;
    int ties = 0;
    if (want) {
        const uint32_t differ = top ^ low;
        int bit = differ ? 31 - __builtin_clz(differ) : -1;
        t = bit < 0 ? top : top & ~((2u << bit) - 1u);
        bool fits = false;
        for (; bit >= 0 && !fits; --bit) {
            const uint32_t c = t | 1u << bit;
            const int n = over_row(count(c));
            if (n >= want) t = c;
            fits = n == want;
        }
        ties = fits ? 0x7fffffff : want - over_row(count(t + 1));   // (no score is 2^32 - 1)
    }
    const unsigned long long below = (1ull << lane) - 1;
    auto kept = [&](int p) { return p < seen && (p < from || p >= to); };
    int at = 0;
    if (W > 1) {   // what the waves before take
        int taken = 0, same = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            same += __builtin_popcountll(__ballot(want && key[n] == t));
            taken += __builtin_popcountll(__ballot(kept(page0 + 64 * n) || (want && key[n] > t)));
        }
        turn ^= 1;
        if (lane == 0) sh.count[turn][wave] = taken, sh.same[wave] = same;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < wave) {
                at += sh.count[turn][w] + min(ties, sh.same[w]);
                ties -= min(ties, sh.same[w]);
            }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int p = page0 + 64 * n;
        if (p - lane >= seen) break;
        const unsigned long long same = __ballot(want && key[n] == t);
        const bool take = kept(p) || (want && key[n] > t) || (want && key[n] == t && __builtin_popcountll(same & below) < ties);
        ties -= min(ties, (int)__builtin_popcountll(same));
        const unsigned long long m = __ballot(take);
        if (take) out[at + __builtin_popcountll(m & below)] = p;
        at += __builtin_popcountll(m);
    }
}

template <int N, int W>
__global__ __launch_bounds__(W > kWaves ? 64 * W : kThreads) void page_select_kernel(SelectArgs a)
{
    __shared__ PickLds<W> sh;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const SelectRow row = select_row(a, W == 1 ? blockIdx.x * kWaves + wave : blockIdx.x);
    if (!row.any) return;
    pick_pages<N, W>(a, row.seen, a.scores + row.at * a.score_stride, a.selected + row.at * a.n_select, W == 1 ? 0 : wave, sh);
}

// Small calls: a block a request and KV head forms the scores of its rows, of no more than
// four tiles, in LDS, and a wave of it a row's list, so that there is one launch and no way
// through memory.
constexpr int kPickWaves = 16;
constexpr int kPickPages = 512;
constexpr int64_t kPickBlocks = 256;   // (of more, each compute unit would have several blocks in turn)

template <bool E4M3, int NC, int R>
__global__ __launch_bounds__(64 * kPickWaves) void page_pick_kernel(SelectArgs a)
{
    extern __shared__ __align__(16) int32_t s_scores[];   // [token][score_stride]
    __shared__ __align__(16) RowsLds<NC, R> sh;
    __shared__ PickLds<1> pick;   // (a wave has no use for it)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r = blockIdx.x / (uint32_t)a.heads;
    const int h = (int)(blockIdx.x - (uint32_t)r * (uint32_t)a.heads);
    const Request rq = request_of(a, r);
    if (rq.rows == 0) return;
    const int most_seen = pages_seen(a, rq, rq.rows - 1);   // (later tokens see no fewer)
    if (most_seen > a.n_select) {
        const int tiles = (most_seen + 15) >> 4;
        score_block<E4M3, NC, R, false, kPickWaves>(a, rq, r, h, 0, most_seen, wave, kPickWaves, max((tiles - wave + kPickWaves - 1) / kPickWaves, 0),
                                                    sh, [&](int tok, int page, int4_t x, bool) { *(int4_t*)(s_scores + tok * a.score_stride + page) = x; });
        __syncthreads();
    }
    int32_t* out = a.selected + (rq.start * (int64_t)a.heads + h) * a.n_select;
    for (int tok = wave; tok < rq.rows; tok += kPickWaves)
        pick_pages<kPickPages / 64, 1>(a, pages_seen(a, rq, tok), s_scores + tok * a.score_stride, out + (int64_t)tok * a.heads * a.n_select, 0, pick);
}

// A block a row, for more pages than a wave holds: digits of 8 bits from the first
// bit that the scores differ in, each from a histogram of those that share the digits
// before.
constexpr int kWideThreads = 1024;

__global__ __launch_bounds__(kWideThreads) void page_select_wide_kernel(SelectArgs a)
{
    constexpr int kWideWaves = kWideThreads / 64;
    __shared__ uint32_t s_count[256];
    __shared__ uint32_t s_top[kWideWaves], s_low[kWideWaves];
    __shared__ int s_before[kWideWaves], s_same[kWideWaves];
    __shared__ uint32_t s_digit, s_left;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const SelectRow row = select_row(a, blockIdx.x);
    if (!row.any) return;
    int32_t* out = a.selected + row.at * a.n_select;
    if (row.seen <= a.n_select) {
        for (int j = tid; j < a.n_select; j += kWideThreads) out[j] = j < row.seen ? j : -1;
        return;
    }
    const int from = a.keep_first, to = row.seen - a.keep_last, want = a.n_select - a.keep_first - a.keep_last;
    const int32_t* scores = a.scores + row.at * a.score_stride;
    auto key_of = [&](int p) { return p >= from && p < to ? key_of_score(scores[p]) : 0u; };
    uint32_t top = 0, low = 0xffffffffu;
    for (int p = tid; p < row.seen; p += kWideThreads) {
        const uint32_t k = key_of(p);
        top = max(top, k);
        low = min(low, k ? k : 0xffffffffu);
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        top = max(top, (uint32_t)__shfl_xor((int)top, k, 64));
        low = min(low, (uint32_t)__shfl_xor((int)low, k, 64));
    }
    if (lane == 0) s_top[wave] = top, s_low[wave] = low;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) top = max(top, s_top[w]), low = min(low, s_low[w]);

    uint32_t t = 0xffffffffu;
    int ties = 0;
    if (want) {
        const uint32_t differ = top ^ low;
        int bits = differ ? 32 - __builtin_clz(differ) : 0;   // still open
        t = bits == 32 ? 0 : top >> bits << bits;
        int left = want;                                      // wanted of those that share the bits settled
        while (bits > 0) {
            const int shift = max(bits - 8, 0), n_digits = 1 << (bits - shift);
            if (tid < 256) s_count[tid] = 0;
            __syncthreads();
            for (int p = tid; p < row.seen; p += kWideThreads) {
                const uint32_t k = key_of(p);
                if (k && ((k ^ t) >> 1 >> (bits - 1)) == 0) atomicAdd(&s_count[(k >> shift) & (uint32_t)(n_digits - 1)], 1u);
            }
            __syncthreads();
            if (wave == 0) {
                // four digits a lane, the largest first; the sum over larger ones says where `left` is reached
                uint32_t c[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c[e] = s_count[255 - (4 * lane + e)];
                    sum += c[e];
                }
                uint32_t upto = sum;
#pragma unroll
                for (int k = 1; k < 64; k <<= 1) {
                    const uint32_t u = __shfl_up(upto, k, 64);
                    if (lane >= k) upto += u;
                }
                uint32_t before = upto - sum;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (before < (uint32_t)left && before + c[e] >= (uint32_t)left) {
                        s_digit = 255 - (4 * lane + e);
                        s_left = (uint32_t)left - before;
                    }
                    before += c[e];
                }
            }
            __syncthreads();
            t |= s_digit << shift;
            left = (int)s_left;
            bits = shift;
            __syncthreads();
        }
        ties = left;
    }
    // the list, 1024 pages at a time
    int at = 0, same_before = 0;
    const unsigned long long below = (1ull << lane) - 1;
    for (int p0 = 0; p0 < row.seen; p0 += kWideThreads) {
        const int p = p0 + tid;
        const uint32_t k = key_of(p);
        const unsigned long long same = __ballot(want && k == t);
        if (lane == 0) s_same[wave] = __builtin_popcountll(same);
        __syncthreads();
        int rank = same_before + __builtin_popcountll(same & below);
#pragma unroll
        for (int w = 0; w < kWideWaves; ++w) {
            if (w < wave) rank += s_same[w];
            same_before += s_same[w];
        }
        const bool kept = p < row.seen && (p < from || p >= to);
        const bool take = kept || (want && k > t) || (want && k == t && rank < ties);
        const unsigned long long m = __ballot(take);
        if (lane == 0) s_before[wave] = __builtin_popcountll(m);
        __syncthreads();
        int mine = at + __builtin_popcountll(m & below);
#pragma unroll
        for (int w = 0; w < kWideWaves; ++w) {
            if (w < wave) mine += s_before[w];
            at += s_before[w];
        }
        if (take) out[mine] = p;
    }
}

// ----------------------------------------------------- attention to lists --

// A tile is four groups of 16 keys of the listed pages; its order of work is that of
// few_keys.  Single tokens' lists come from memory (16 requests with 64 pages of 64 x 128, 8
// heads: 135 MB in 26 us, 5.1 TB/s).  Lists that many tokens share come from the caches, and
// what bounds them is the vector unit (a chunk of 4096 tokens with 16 pages each: 500 us, 0.14
// PFLOP/s, the unit 89% busy; 192 of a tile's some 325 instructions widen int8 codes to binary16, once for each token:
// lists differ): so a weight with its value scale is one power of two,
// 2^(s c - m + log2 v), as in the kernel for many rows: v = vs 2^8 / vr is held at 2^-40 from
// below, and a sum over v is what l wants.
//
// SHIFTED, of int8 codes where the vector unit is what a call waits for: codes are taken as 2^-24 (c + 128), a byte each as a
// subnormal binary16 number, three instructions for four codes in place of five (the chunk 580 -> 513 us).  What the 128 add is
// taken out of the sums: of a score's by where it begins, of the values' tile by tile, by 128 times the sum of the tile's weights
// as they were rounded.  (Once at the end it is 499 us, but the sums then grow with the list, and with them their roundings: an
// error of 2^-15 of a code's step at 16 tiles, 2^-12 at 512.)  So a score's roundings are of sums of up to 255 units where they
// had |c|, and the values' are, beside those of the sums themselves, four a tile of up to 255 units of that tile's weights: one
// rounding a product, 2^-14 of a step at most over a list of any length, 2^-18 as emulated, and a step stands for anything within
// half of it.
__device__ __forceinline__ half8_t shifted8(uint32_t a, uint32_t b)
{
    const uint32_t x = a ^ 0x80808080u, y = b ^ 0x80808080u;
    return __builtin_bit_cast(half8_t, make_uint4(__builtin_amdgcn_perm(0, x, 0x0c010c00u), __builtin_amdgcn_perm(0, x, 0x0c030c02u),
                                                  __builtin_amdgcn_perm(0, y, 0x0c010c00u), __builtin_amdgcn_perm(0, y, 0x0c030c02u)));
}

template <bool E4M3, bool SHIFTED>
__device__ __forceinline__ half8_t listed8(uint32_t a, uint32_t b)
{
    if constexpr (SHIFTED) return shifted8(a, b);
    else return codes8<E4M3>(a, b);
}

template <int NC, bool SHIFTED>
struct ListedQuery : FewQuery<NC> {
    float4_t base;   // of a row's products
    __device__ __forceinline__ ListedQuery(const AttendArgs& a, const Request& rq, const FewRow& fr) : FewQuery<NC>(a, rq, fr), base{0, 0, 0, 0}
    {
        // a negative scale's sign goes into the row, so that the factor of a score is not negative
        const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u;
        this->mul = fabsf(this->mul);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint4 u = __builtin_bit_cast(uint4, this->qf[c][k]);
                u.x ^= sign, u.y ^= sign, u.z ^= sign, u.w ^= sign;
                this->qf[c][k] = __builtin_bit_cast(half8_t, u);
            }
        if constexpr (SHIFTED) {
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += (float)this->qf[c][k][e];
            sum = rows_sum(sum) * -0x1p-17f;   // 128 x 2^-24
            base = float4_t{sum, sum, sum, sum};
        }
    }
};

template <bool E4M3, int NC, bool SHIFTED>
__device__ __forceinline__ void listed_products(const uint4 (&kw)[4][NC], const ListedQuery<NC, SHIFTED>& q, float4_t (&s)[4])
{
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        s[t] = q.base;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(listed8<E4M3, SHIFTED>(kw[t][c].x, kw[t][c].y), q.qf[c][0], s[t], 0, 0, 0);
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(listed8<E4M3, SHIFTED>(kw[t][c].z, kw[t][c].w), q.qf[c][1], s[t], 0, 0, 0);
        }
    }
}

// PLAIN: neither cap nor bias.  U: of few rows the operands' 16 columns hold each U times
// over, and column u of a row's takes the u-th part of every 16 keys, as a wave of its own
// would: its weights are 0 elsewhere.  (Of groups of four the chunk took 632 us without and 619 with it; where a block's waves
// are joined in LDS, four times the parts cost one token over 32 pages 1 of 16 us.)
template <bool E4M3, int NC, bool PLAIN, int U, bool SHIFTED>
__device__ __forceinline__ void listed_update(const AttendArgs& a, const Request& rq, const Seen& mine, const ListedQuery<NC, SHIFTED>& q,
                                              FewSums<NC>& st, float4_t (&s)[4], uint4 (&vw)[4 * NC], float2 sc, bool here, bool mask, int j0g)
{
    constexpr int N = 16 / U;   // keys
    const int u = (threadIdx.x & 15) / N;
    const int j0 = j0g + u * N;
    float c = q.mul * sc.x;   // a score's factor
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = s[i >> 2][i & 3];
#pragma unroll
        for (int k = 1; k < U; ++k) x[i] = u == k ? s[(k * N + i) >> 2][i & 3] : x[i];
    }
    if (SHIFTED) {   // the codes' 2^24 goes into the factor, or into the products where that would be beyond fp32's end
        if (__any(c > 0x1p100f)) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] *= 0x1p24f;
        } else {
            c *= 0x1p24f;
        }
    }
    c = fmaxf(c, 0x1p-120f);   // (never 0: hidden scores are infinite)
    if (!PLAIN && (q.cap > 0.0f || q.slopes)) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= c;
        if (q.large_cap) {
            const float inv = 1.0f / q.cap2;
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = capped_large(x[i], q.cap2, inv);
        } else if (q.cap > 0.0f) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = capped(x[i], q.cap2);
        }
        if (q.slopes) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] -= q.slope2 * fabsf((float)(j0 + i - q.pos));
        }
        c = 1.0f;
    }
    if (mask) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!here || !visible(a, mine, j0 + i)) x[i] = -__builtin_inff();
        if (E4M3) {   // codes after the last key may be anything, a NaN among it
            const int n = here ? rq.kv - j0g : 0;
#pragma unroll
            for (int t = 0; t < 4 * NC; ++t) vw[t] = first_bytes(vw[t], n);
        }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = __builtin_elementwise_maximum(top, x[i]);
    const float vtop = top > -__builtin_inff() ? sc.y : 0.0f;   // of a group of which the column sees a key
    top = rows_max(top * c);
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
    const float v = __builtin_amdgcn_fmed3f(sc.y * (kTop * __builtin_amdgcn_rcpf(st.vref)), 0x1p-40f, kTop);   // (more only where all weights are 0)
    const float log_v = __builtin_amdgcn_logf(v);
    float vb = log_v - m0;
    // the product of a large score is rounded before the maximum is taken off, as it was for that: exact, it may be far above
    if (__any(fabsf(m0) > 0x1p20f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = x[i] * c - m0;
        c = 1.0f;
        vb = log_v;
    }
    uint32_t p[8];   // the 16 keys' weights
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, vb)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i + 1], c, vb));
        sum += w0;
        sum += w1;
        const half2_t two = {(_Float16)w0, (_Float16)w1};
#pragma unroll
        for (int k = 0; k < U; ++k) p[(k * N + i) / 2] = U == 1 || u == k ? __builtin_bit_cast(uint32_t, two) : 0u;
    }
    st.l = __builtin_fmaf(sum, __builtin_amdgcn_rcpf(v), st.l);
    const half8_t p0 = __builtin_bit_cast(half8_t, make_uint4(p[0], p[1], p[2], p[3]));
    const half8_t p1 = __builtin_bit_cast(half8_t, make_uint4(p[4], p[5], p[6], p[7]));
    if constexpr (SHIFTED) {   // the tile's 128 out of the sums: 2^-24 x 128 times the weights as they were rounded
        const half8_t ones = {1, 1, 1, 1, 1, 1, 1, 1};
        float4_t weights = {0, 0, 0, 0};
        weights = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p0, weights, 0, 0, 0);
        weights = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p1, weights, 0, 0, 0);
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.acc[t][e] = __builtin_fmaf(weights[e], -0x1p-17f, st.acc[t][e]);
    }
#pragma unroll
    for (int t = 0; t < 4 * NC; ++t) {
        st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(listed8<E4M3, SHIFTED>(vw[t].x, vw[t].y), p0, st.acc[t], 0, 0, 0);
        st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(listed8<E4M3, SHIFTED>(vw[t].z, vw[t].w), p1, st.acc[t], 0, 0, 0);
    }
}

// Where the 16-key group at place `at` of a list of pages lies, whose entry there is
// known: `pos` is its first key.  Pages of entries that are no column of the request's
// are not there.
struct ListPlace : Place {
    int pos;
};

__device__ __forceinline__ int list_entry(const AttendArgs& a, int at)   // the list's entry that holds place `at`
{
    return a.per_page_inv ? (int)__umulhi((uint32_t)at, a.per_page_inv) : at;
}

__device__ __forceinline__ ListPlace place_listed(const AttendArgs& a, const int32_t* table, int kv, int places, int at, int column)
{
    ListPlace p;
    p.in_page = at - list_entry(a, at) * (int)a.per_page;
    const int last = (kv - 1) >> 4;   // kv >= 1
    const int columns = (int)((a.per_page_inv ? __umulhi((uint32_t)last, a.per_page_inv) : (uint32_t)last) + 1);
    p.here = at < places && (uint32_t)column < (uint32_t)columns;
    column = p.here ? column : 0;
    p.pos = (column * (int)a.per_page + p.in_page) * 16;
    p.id = table[column];
    return p;
}

// A wave over the tiles e0, e0 + step, .. below e1 (one at least) of a list of `places`
// groups, for rows of one token.  Any pages: a lane group looks up its own group's.  The
// entries are read two tiles ahead, the pages' ids one.
template <bool E4M3, int NC, bool PLAIN, int U, bool SHIFTED>
__device__ __forceinline__ void listed_groups(const AttendArgs& a, const Request& rq, int64_t r, int h, const FewRow& fr, int e0, int step,
                                              int e1, FewSums<NC>& st, const int32_t* list, int places)
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
    auto load_keys = [&](const Place& p) {
        const uint8_t* kp = k_head + p.id * per_id + p.in_page * 16 * d;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) kw[t][c] = *(const uint4*)(kp + kc[c] + t * 4 * d);
    };
    auto entry = [&](int e, int k) { return list[list_entry(a, min(4 * min(e, e1 - 1) + k, places - 1))]; };
    auto place = [&](int e, int k, int column) { return place_listed(a, table, rq.kv, places, 4 * min(e, e1 - 1) + k, column); };
    const int ck0 = entry(e0, gk), cv0 = entry(e0, g), ck1 = entry(e0 + step, gk), cv1 = entry(e0 + step, g);
    int ck2 = entry(e0 + 2 * step, gk), cv2 = entry(e0 + 2 * step, g);
    ListPlace pk = place(e0, gk, ck0), pv = place(e0, g, cv0);
    ListPlace pk1 = place(e0 + step, gk, ck1), pv1 = place(e0 + step, g, cv1);
    check_place(a, pk);
    check_place(a, pv);
    load_keys(pk);
    float2 sc = scale_head[(int64_t)pv.id * a.heads], sc_next = sc;
    const ListedQuery<NC, SHIFTED> query(a, rq, fr);
    for (int e = e0; e < e1; e += step) {
        // the tile's values, on their way while its scores are formed
        uint4 vw[4 * NC];
        const uint8_t* vp = v_head + pv.id * per_id + pv.in_page * 16 * d;
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) vw[t] = *(const uint4*)(vp + min(t * 16, d - 16) * 16);
        const bool here = pv.here;
        const int j0g = pv.pos;
        const bool mask = __any(!here || j0g < mine.lo || j0g + 16 > mine.hi || (a.window && j0g < mine.wlo && j0g + 16 > a.sinks));
        if (!here) sc = make_float2(0.0f, 0.0f);
        float4_t s[4];
        listed_products<E4M3, NC>(kw, query, s);
        // the next tile's keys, and the pages and entries of those after
        if (e + step < e1) {
            check_place(a, pk1);
            check_place(a, pv1);
            load_keys(pk1);
            sc_next = scale_head[(int64_t)pv1.id * a.heads];
            pv = pv1;
            pk1 = place(e + 2 * step, gk, ck2);
            pv1 = place(e + 2 * step, g, cv2);
            ck2 = entry(e + 3 * step, gk);
            cv2 = entry(e + 3 * step, g);
        }
        listed_update<E4M3, NC, PLAIN, U, SHIFTED>(a, rq, mine, query, st, s, vw, sc, here, mask, j0g);
        sc = sc_next;
    }
    st.l = rows_sum(st.l);
}

template <int NC> constexpr int kKeyBytes = 4 * NC * 1024;   // of a wave's LDS

// A tile's keys in LDS, 64 rows of d / 16 16-byte chunks, on their way there without registers: a left operand takes 16 rows
// at a time, of which no two lie in a line, and read from memory so a load holds the cache's address unit for 64 cycles, not 16
// (a chunk of 4096 tokens with lists of 16 pages of 64 x 128, 8 heads: the unit 93% busy and 620 us, so 570).  A row's chunks are
// turned by a number of places so that 16 rows' reads fall into different banks.
template <int NC>
struct KeyTile {
    uint8_t* lds;
    uint32_t from[4 * NC];   // where in the tile this lane's 16 bytes of a load lie
    uint32_t at[NC];         // its first operand's chunk in LDS
    uint32_t chunks;
    __device__ __forceinline__ KeyTile(uint8_t* lds_, int d) : lds(lds_), chunks(d >> 4)
    {
        const uint32_t lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
        auto places = [&](uint32_t row) {
            const uint32_t n = NC == 1 ? row >> 4 : NC == 2 ? (row >> 1 & 1) + 2 * (row >> 4) : (row & 3) + 4 * (row >> 4);
            return n < chunks ? n : 0;
        };
        uint32_t to_row = lane / chunks, to = lane - to_row * chunks;
        const uint32_t rows = 64 / chunks, rest = 64 - rows * chunks;
#pragma unroll
        for (int i = 0; i < 4 * NC; ++i) {
            const uint32_t source = min(to_row, 63u), n = places(source);   // (rows of fewer than 4 NC chunks: some loads for nothing)
            from[i] = (source * chunks + (to >= n ? to - n : to + chunks - n)) * 16;
            to_row += rows;
            to += rest;
            if (to >= chunks) to -= chunks, ++to_row;
        }
        const uint32_t row = (c16 >> 2) * 16 + (c16 & 3), n = places(row);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint32_t chunk = min(4 * c + g, chunks - 1) + n;   // channels beyond d are taken from the last ones: q is zero there
            at[c] = (row * chunks + (chunk >= chunks ? chunk - chunks : chunk)) * 16;
        }
    }
    __device__ __forceinline__ void fetch(const uint8_t* keys) const
    {
#pragma unroll
        for (int i = 0; i < 4 * NC; ++i) {
            uint32_t offset = from[i];
            asm("" : "+v"(offset));   // (32 bits beside an address in scalar registers)
            __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(keys + offset),
                                             (void __attribute__((address_space(3)))*)(lds + i * 1024), 16, 0, 0);
        }
    }
    __device__ __forceinline__ void read(uint4 (&kw)[4][NC]) const
    {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // fetched
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) kw[t][c] = *(const uint4*)(lds + at[c] + t * 64 * chunks);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // and read: the next ones may come
    }
};

// The same of pages of a multiple of 64 tokens: a tile lies in one page, so
// that its place and scales are the same in all lanes; they are looked up in scalar
// registers, and the loads of codes take their addresses from there and from offsets that
// stay as they are.  The entries are read two tiles ahead, the pages' ids and scales one.
// THROUGH: the keys go through LDS; where few items wait for their tiles in turn the way
// there is longer than it is worth (16 requests with 64 pages each, 8 heads: 34.2 us, 32.9).
template <bool E4M3, int NC, bool PLAIN, int U, bool THROUGH, bool SHIFTED>
__device__ __forceinline__ void whole_tiles(const AttendArgs& a, const Request& rq, int64_t r, int h, const FewRow& fr, int e0, int step,
                                            int e1, FewSums<NC>& st, const int32_t* list, uint8_t* lds)
{
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int d = a.d;
    const int64_t per_head = (int64_t)a.page * d;
    Seen mine = seen_of(a, rq, r, fr.tok);   // (rows of one token: alike in all lanes)
    mine.lo = __builtin_amdgcn_readfirstlane(mine.lo);
    mine.hi = __builtin_amdgcn_readfirstlane(mine.hi);
    mine.wlo = __builtin_amdgcn_readfirstlane(mine.wlo);
    const int32_t* table = a.tables + r * a.max_pages;
    const uint32_t columns = (uint32_t)pages_of(a, rq.kv);
    // (an offset of 32 bits beside an address in scalar registers, as loads take them; widened outside of the loop, each
    // load would have an address of its own in vector registers)
    auto here_of = [](uint32_t offset) {
        asm("" : "+v"(offset));
        return offset;
    };
    struct Tile {
        int64_t at;   // its codes, of keys as of values
        float2 scales;
        int pos;
        bool here;
    };
    struct Place {
        int id, pos, in_page;   // in_page: 16-token groups
        bool here;
    };
    auto column = [&](int e) { return scalar_load(list + list_entry(a, 4 * min(e, e1 - 1))); };
    auto place = [&](int e, int col) {
        Place p;
        const int at = 4 * min(e, e1 - 1);
        p.in_page = at - list_entry(a, at) * (int)a.per_page;
        p.here = (uint32_t)col < columns;
        col = p.here ? col : 0;
        p.pos = (col * (int)a.per_page + p.in_page) * 16;
        p.id = scalar_load(table + col);
        return p;
    };
    auto tile_of = [&](const Place& p) {
        Tile t;
        t.here = p.here && (uint32_t)p.id < (uint64_t)a.n_pages;
        const int64_t of_head = (t.here ? p.id : 0) * (int64_t)a.heads + h;
        t.at = of_head * per_head + p.in_page * 16 * d;
        t.scales = __builtin_bit_cast(float2, scalar_load((const uint64_t*)(a.scales + of_head)));
        t.pos = p.pos;
        return t;
    };
    // channels beyond d are loaded from the last ones: q is zero there, and their sums go nowhere
    uint32_t kc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) kc[c] = (c16 >> 2) * 16 * d + (c16 & 3) * d + min(c * 64 + g * 16, d - 16);
    const uint32_t vc = g * 16 * d + c16 * 16;
    const KeyTile<NC> keys(lds, d);
    uint4 kw[4][NC], vw[4 * NC];
    auto load_keys = [&](const Tile& t) {
        const uint8_t* kp = a.k_codes + t.at;
        if constexpr (THROUGH) {
            keys.fetch(kp);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < NC; ++c) kw[i][c] = *(const uint4*)(kp + i * 4 * d + here_of(kc[c]));
        }
    };
    auto load_values = [&](const Tile& t) {
        const uint8_t* vp = a.v_codes + t.at;
#pragma unroll
        for (int i = 0; i < 4 * NC; ++i) vw[i] = *(const uint4*)(vp + min(i * 16, d - 16) * 16 + here_of(vc));
    };
    const int c0 = column(e0), c1 = column(e0 + step);
    int c2 = column(e0 + 2 * step);
    const Place p0 = place(e0, c0);
    Place next = place(e0 + step, c1);
    Tile now = tile_of(p0);
    load_keys(now);
    const ListedQuery<NC, SHIFTED> query(a, rq, fr);
    for (int e = e0; e < e1; e += step) {
        const Tile tile = now;
        auto advance = [&] {
            now = tile_of(next);   // (behind the last tile that one again, but its keys)
            if (e + step < e1) load_keys(now);
            next = place(e + 2 * step, c2);
            c2 = column(e + 3 * step);
        };
        float4_t s[4];
        if constexpr (THROUGH) {   // (loads arrive in their order: the next tile's keys first, and with the values they are there)
            keys.read(kw);
            advance();
            load_values(tile);
            listed_products<E4M3, NC>(kw, query, s);
        } else {
            load_values(tile);
            listed_products<E4M3, NC>(kw, query, s);
            advance();
        }
        const bool mask = !tile.here || tile.pos < mine.lo || tile.pos + kTile > mine.hi || (tile.pos < mine.wlo && tile.pos + kTile > a.sinks);
        const float2 sc = tile.here ? tile.scales : make_float2(0.0f, 0.0f);
        listed_update<E4M3, NC, PLAIN, U, SHIFTED>(a, rq, mine, query, st, s, vw, sc, tile.here, mask, tile.pos + g * 16);
    }
    st.l = rows_sum(st.l);
}

// W waves an item -- a token, a KV head and up to 16 of its query heads -- that take
// the list's tiles in turn, with those of the item's other splits; their sums joined
// in LDS, and the splits' by a second kernel.
template <bool E4M3, int NC, int W, bool WHOLE, bool PLAIN, int U>
__global__ __launch_bounds__(W > kWaves ? 64 * W : kThreads, NC == 2 && WHOLE && W <= kWaves ? 3 : NC <= 2 ? 2 : 1) void attend_listed_kernel(AttendArgs a)
{
    extern __shared__ __align__(16) float lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    constexpr int kColumns = kFewRows / U;   // that hold the rows once
    const int d = a.d, row = c16 & (kColumns - 1);
    const int64_t q_heads = (int64_t)a.heads * a.group;
    const int split = (int)(blockIdx.x % (uint32_t)a.n_splits);
    const uint32_t block = blockIdx.x / (uint32_t)a.n_splits;
    const uint32_t chunks = (uint32_t)(a.group + kFewRows - 1) / kFewRows;
    // (blocks of one head go to one part of the chip, where the heads are as many as its parts: a head's pages are read there
    // more often.  A wave an item: neighbouring tokens of one head in a block)
    const uint32_t of_head = block / (uint32_t)a.heads;
    const int h = (int)(block - of_head * (uint32_t)a.heads);
    const uint32_t of_chunk = of_head / chunks;
    const int chunk = (int)(of_head - of_chunk * chunks);
    const int64_t ri = W == 1 ? (int64_t)of_chunk * kWaves + wave : of_chunk;
    if (ri >= (a.searched ? a.searched : a.n_req * a.max_new)) return;
    const TokenPlace at = token_place(a, (uint32_t)ri);
    if (at.r < 0) return;
    const int64_t r = at.r;
    const Request rq = request_of(a, r);
    const int i = at.i < 0 ? (int)ri - rq.start : at.i;
    if ((uint32_t)i >= (uint32_t)rq.rows) return;   // (negative: of starts out of order)
    const int64_t token = rq.start + i;
    const int32_t* list = a.listed + (token * a.heads + h) * a.n_listed;
    int n = 0;   // entries up to the last that names a page
    if (rq.kv > 0)
        for (int j0 = 0; j0 < a.n_listed; j0 += 64) {
            const unsigned long long m = __ballot(j0 + lane < a.n_listed && list[min((int64_t)(j0 + lane), a.n_listed - 1)] >= 0);
            if (m) n = j0 + 64 - __builtin_clzll(m);
        }
    const int places = n * (int)a.per_page, tiles = (places + 3) >> 2;
    const int n_rows = min(a.group - chunk * kFewRows, kFewRows);
    const FewRow fr = {min(row, n_rows - 1), i, h * a.group + chunk * kFewRows + min(row, n_rows - 1)};
    constexpr bool kShifted = !E4M3 && W == 1;
    FewSums<NC> st;
    const int e0 = split * W + (W == 1 ? 0 : wave);
    if (e0 < tiles) {
        if constexpr (WHOLE) whole_tiles<E4M3, NC, PLAIN, U, W == 1, kShifted>(a, rq, r, h, fr, e0, a.n_splits * W, tiles, st, list, (uint8_t*)lds + wave * kKeyBytes<NC>);
        else listed_groups<E4M3, NC, PLAIN, U, kShifted>(a, rq, r, h, fr, e0, a.n_splits * W, tiles, st, list, places);
    }

    if (kShifted) {
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) st.acc[t] *= 0x1p24f;
    }
    if (W == 1) {
        if (U > 1) {   // a row's columns together
            auto over_columns = [](float x, auto join) {
                x = join(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xf, 0xf, false)));   // 8 lanes on
                if (U > 2) x = join(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x124, 0xf, 0xf, false)));
                return x;
            };
            auto sum = [](float x, float y) { return x + y; };
            auto most = [](float x, float y) { return fmaxf(x, y); };
            const float m = over_columns(st.m, most), vref = over_columns(st.vref, most);
            const float k = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(st.m - m);
            st.l = over_columns(st.l * k, sum);
            const float kv = k * (st.vref / vref);
#pragma unroll
            for (int t = 0; t < 4 * NC; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.acc[t][e] = over_columns(st.acc[t][e] * kv, sum);
            st.m = m;
            st.vref = vref;
        }
        if (c16 >= n_rows) return;
        const float inv = st.l == 0.0f ? 0.0f : st.vref * (1.0f / kTop) / st.l;
#pragma unroll
        for (int t = 0; t < 4 * NC; ++t) {
            const float4_t o = st.acc[t] * inv;
            if (t * 16 < d)
                *(uint2*)(a.out + 2 * (token * a.o_token + fr.head * a.o_head + t * 16 + g * 4)) =
                    make_uint2(f32_to_row2(o[0], o[1], a.bf16), f32_to_row2(o[2], o[3], a.bf16));
        }
        if (g == 0 && a.lse) a.lse[token * q_heads + fr.head] = st.l == 0.0f ? -__builtin_inff() : kLn2 * (st.m + __log2f(st.l));
        return;
    }
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
        const int64_t hq = h * a.group + chunk * kFewRows + rw;
        if (a.n_splits > 1) {
            const int64_t at = (token * q_heads + hq) * a.n_splits + split;
            *(float4_t*)(a.part + at * d + 4 * q4) = o;
            if (q4 == 0) a.stat[at] = make_float2(mm, ll);
            continue;
        }
        const float inv = ll == 0.0f ? 0.0f : (1.0f / kPart) / ll;
        *(uint2*)(a.out + 2 * (token * a.o_token + hq * a.o_head + 4 * q4)) =
            make_uint2(f32_to_row2(o[0] * inv, o[1] * inv, a.bf16), f32_to_row2(o[2] * inv, o[3] * inv, a.bf16));
        if (q4 == 0 && a.lse) a.lse[token * q_heads + hq] = ll == 0.0f ? -__builtin_inff() : kLn2 * (mm + __log2f(ll));
    }
}

// ------------------------------------------------------------------ host --

constexpr int64_t kMostBlocks = 0x7fffff00;
constexpr int64_t kMostListed = 1 << 20;

bool select_ok(const fkv_page_desc* p, const fkv_select_desc* t)
{
    constexpr int64_t kMost = 1 << 30;
    return page_desc_ok(p) && t && t->n_req >= 0 && t->n_req <= kMost && t->n_tokens >= 0 && t->n_tokens <= kMost &&
           t->max_new >= 1 && t->max_new <= kMost && t->max_kv >= 0 && t->max_kv <= kMost && t->max_pages >= 1 &&
           t->max_pages <= (1 << 26) && stride_ok(t->q_stride_token) && stride_ok(t->q_stride_head) && t->q_heads >= 1 &&
           t->q_heads <= 65535 && t->q_heads % p->heads == 0 && (t->type == FKV_ROW_F16 || t->type == FKV_ROW_BF16) &&
           (t->causal == 0 || t->causal == 1) && t->n_select >= 1 && t->n_select <= kMostListed && t->keep_first >= 0 &&
           t->keep_last >= 0 && (int64_t)t->keep_first + t->keep_last <= t->n_select;
}

// Pages that a request may have, and a row of scores: none where every page is selected.
int64_t most_pages(const fkv_page_desc* p, const fkv_select_desc* t)
{
    return std::min((t->max_kv + p->page - 1) / p->page, t->max_pages);
}

int64_t score_stride(const fkv_page_desc* p, const fkv_select_desc* t)
{
    const int64_t n = most_pages(p, t);
    return n <= t->n_select ? 0 : (n + 15) / 16 * 16;
}

// a * b, or the largest size there is: of sizes beyond any memory.
size_t bytes_or_most(size_t a, size_t b)
{
    size_t n;
    return __builtin_mul_overflow(a, b, &n) ? ~(size_t)0 : n;
}

int lanes_log(int64_t group)
{
    int n = 0;
    while (n < 4 && (1 << n) < group) ++n;
    return n;
}

// Whether page_pick_kernel does a call.  Without and with it (us a call, with the host's part): a token over 512 pages, 8 KV heads
// of 128 16.0 and 11.8, 16 such requests 16.8 and 12.4, 8 of four tokens each 16.2 and 11.9.  Of 2048 pages it takes 31 in
// place of 28, and 512 requests of 128 pages 157 in place of 42.
bool picked_at_once(const fkv_page_desc* p, const fkv_select_desc* t)
{
    const int64_t group = t->q_heads / p->heads;
    return score_stride(p, t) && group <= 16 && p->d <= 128 && t->max_new <= 4 * (16 >> lanes_log(group)) && most_pages(p, t) <= kPickPages &&
           t->n_req * p->heads <= kPickBlocks;
}

constexpr int kHeldPages = 16384;   // that the waves of a row hold at the most: 16 of 16 x 64

// Places for tokens in a launch, and whether their requests are looked up: where that spares half of them.
int64_t searched_rows(int64_t n_req, int64_t max_new, int64_t n_tokens)
{
    n_tokens = std::max(n_tokens, (int64_t)1);
    return n_req * max_new >= 2 * n_tokens ? n_tokens : 0;
}

struct ListedShape {
    int waves;       // of an item in a block
    int n_splits;
    int64_t blocks;  // times the splits
    int64_t searched;
    bool join_blocks;
};

ListedShape listed_shape(const fkv_page_desc* p, const fkv_attend_desc* t, int64_t n_listed)
{
    ListedShape s;
    const int64_t group = t->q_heads / p->heads;
    const int64_t of_token = p->heads * ((group + kFewRows - 1) / kFewRows);
    s.searched = searched_rows(t->n_req, t->max_new, t->n_tokens);
    const int64_t tokens = s.searched ? s.searched : t->n_req * t->max_new;   // below 2^31
    const int64_t items = tokens * of_token;
    const int64_t tiles = (n_listed * (p->page / 16) + 3) / 4;
    // A wave an item where the items fill the chip, else four.  Of few items with up to 32 tiles eight waves have up to four tiles
    // each and no second launch; longer lists are split, two tiles a wave at the least.  Measured with four waves, eight, and
    // four splits of four (us a call, with the host's part), 8 KV heads of 128: one token, 16 tiles 14.6, 14.5 and 19.1, 32 tiles
    // 18.2, 17.0 and 19.0, 64 tiles 30, 27 and 19.3; 16 tokens, 32 tiles 21.2, 19.6 and 21.0, 64 tiles 38, 33 and 31; 32 tokens,
    // 32 tiles 26.3, 26.5 and 33.1; 64 tokens 54, 58 and 63.
    s.n_splits = 1;
    s.waves = items >= 2048 || tiles <= 1 ? 1 : kWaves;
    s.blocks = s.waves == 1 ? (tokens + kWaves - 1) / kWaves * of_token : items;
    if (items < 256 && tiles > 16 && tiles <= 32 && p->d <= 128) {
        s.waves = 8;
    } else if (items < 256 && tiles > 16) {
        const int64_t want = (512 + items - 1) / std::max((int64_t)1, items), most = std::max((int64_t)1, tiles / (2 * kWaves));
        s.n_splits = (int)std::min(want, most);
    }
    s.join_blocks = s.n_splits >= kManySplits;
    return s;
}

Workspace listed_workspace(const fkv_page_desc* p, const fkv_attend_desc* t, const ListedShape& s)
{
    if (s.n_splits == 1) return Workspace{0, 0, 0};
    const size_t rows = (size_t)(t->n_tokens * t->q_heads) * (size_t)s.n_splits;
    Workspace w;
    w.stat = rows * p->d * sizeof(float);
    w.pieces = w.bytes = bytes_or_most(rows, p->d * sizeof(float) + sizeof(float2));
    return w;
}

}  // namespace
}  // namespace fkv

using namespace fkv;

extern "C" size_t fkv_page_select_workspace(const fkv_page_desc* desc, const fkv_select_desc* select)
{
    if (!select_ok(desc, select) || picked_at_once(desc, select)) return 0;
    return bytes_or_most((size_t)(select->n_tokens * desc->heads), (size_t)score_stride(desc, select) * sizeof(int32_t));
}

extern "C" int fkv_page_select(const fkv_page_desc* desc, const fkv_select_desc* select, const uint8_t* boxes, const float* scales,
                               const void* q, const int32_t* tables, const int32_t* kv_len, const int32_t* q_start,
                               int32_t* selected, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!select_ok(desc, select)) return FKV_ERR_INVALID_ARG;
    if (!boxes || !scales || !aligned(boxes, 16) || !aligned(scales, 8)) return FKV_ERR_INVALID_ARG;
    if (select->n_req == 0 || select->n_tokens == 0) return FKV_OK;
    if (!q || !tables || !kv_len || !q_start || !selected || !aligned(q, 16) || !aligned(tables, 4) || !aligned(kv_len, 4) ||
        !aligned(q_start, 4) || !aligned(selected, 4) || !aligned(workspace, 16))
        return FKV_ERR_INVALID_ARG;
    const size_t need = fkv_page_select_workspace(desc, select);
    if (need && (!workspace || workspace_bytes < need)) return FKV_ERR_SCRATCH_TOO_SMALL;
    fkv_attend_desc t = {};
    t.n_req = select->n_req, t.n_tokens = select->n_tokens, t.max_new = select->max_new, t.max_kv = select->max_kv;
    t.max_pages = select->max_pages, t.q_stride_token = select->q_stride_token, t.q_stride_head = select->q_stride_head;
    t.q_heads = select->q_heads, t.type = select->type, t.causal = select->causal;
    SelectArgs a = {};
    (AttendArgs&)a = attend_args(desc, &t, nullptr, nullptr, scales, q, tables, kv_len, q_start, nullptr, nullptr, nullptr, nullptr, nullptr);
    a.boxes = boxes, a.scores = (int32_t*)workspace, a.selected = selected;
    a.score_stride = score_stride(desc, select);
    a.n_select = select->n_select, a.keep_first = select->keep_first, a.keep_last = select->keep_last;
    const int64_t pages = most_pages(desc, select);
    const hipStream_t st = (hipStream_t)stream;
    a.searched = searched_rows(a.n_req, a.max_new, a.n_tokens);
    const int64_t tokens = a.searched ? a.searched : a.n_req * a.max_new;   // below 2^31
    if (tokens > kMostBlocks / a.heads) return FKV_ERR_UNSUPPORTED;
    const int64_t rows = tokens * a.heads;
    const bool e4m3 = desc->format == FKV_PAGE_E4M3;
    a.lanes_log = lanes_log(a.group);
    if (picked_at_once(desc, select)) {
        auto go = [&](auto kern) {
            hipLaunchKernelGGL(kern, dim3((unsigned)(a.n_req * a.heads)), dim3(64 * kPickWaves), (size_t)(a.max_new * a.score_stride) * sizeof(int32_t), st, a);
        };
        auto of_width = [&](auto nc) {
            constexpr int NC = decltype(nc)::value;
            if (a.max_new <= 16 >> a.lanes_log) return e4m3 ? go(page_pick_kernel<true, NC, 1>) : go(page_pick_kernel<false, NC, 1>);
            e4m3 ? go(page_pick_kernel<true, NC, 4>) : go(page_pick_kernel<false, NC, 4>);
        };
        if (a.d <= 64) of_width(std::integral_constant<int, 1>{});
        else of_width(std::integral_constant<int, 2>{});
        return launch_status();
    }
    if (need) {
        const int64_t row_tiles = (a.max_new + (16 >> a.lanes_log) - 1) / (16 >> a.lanes_log);
        const bool many = a.group > 16 || row_tiles >= 4;   // four row tiles a block
        a.row_groups = a.group > 16 || !many ? row_tiles : (row_tiles + 3) / 4;
        const int64_t per = a.group > 16 ? 1 : (many ? 4 : 1) * (16 >> a.lanes_log);   // tokens of a group
        const int64_t found = a.n_tokens / per + (per > 1 ? a.n_req : 0), in_order = a.n_req * a.row_groups;
        a.searched_groups = in_order >= 2 * found ? found : 0;
        const int64_t groups = a.searched_groups ? found : in_order;   // below 2^32
        const int64_t tiles = (pages + 15) / 16;
        // as many page tiles a wave as leave the chip eight thousand waves, where rounding the rows is to be shared.  With 2
        // and 8 a wave (us): a chunk of 4096 tokens over 512 pages 136 and 104, 512 tokens over 256 pages 20 and 23; few rows,
        // 16 contexts of 2048 pages 28.7 and 28.1, 64 of up to 2048 pages 27 and 34, one of 16,384 pages 32 and 35.
        int64_t wave_tiles = std::min(groups * a.heads, (int64_t)1 << 40) * tiles / 8192;
        wave_tiles = many ? std::min((int64_t)8, std::max((int64_t)2, wave_tiles)) : 2;
        a.wave_tiles = (int32_t)wave_tiles;
        a.tile_chunks = (int32_t)((tiles + wave_tiles * kWaves - 1) / (wave_tiles * kWaves));
        const int64_t blocks = groups * a.heads;
        if (blocks > kMostBlocks / a.tile_chunks) return FKV_ERR_UNSUPPORTED;
        auto go = [&](auto kern) {
            hipLaunchKernelGGL(kern, dim3((unsigned)(blocks * a.tile_chunks)), dim3(kThreads), 0, st, a);
        };
        auto of_width = [&](auto nc) {
            constexpr int NC = decltype(nc)::value;
            if (a.group > 16) return e4m3 ? go(page_score_kernel<true, NC, 4, true>) : go(page_score_kernel<false, NC, 4, true>);
            if (many) return e4m3 ? go(page_score_kernel<true, NC, 4, false>) : go(page_score_kernel<false, NC, 4, false>);
            e4m3 ? go(page_score_kernel<true, NC, 1, false>) : go(page_score_kernel<false, NC, 1, false>);
        };
        if (a.d <= 64) of_width(std::integral_constant<int, 1>{});
        else if (a.d <= 128) of_width(std::integral_constant<int, 2>{});
        else of_width(std::integral_constant<int, 4>{});
    }
    // a wave a row where the rows are many, four where they leave the chip idle, 16 for more pages
    auto held = [&](auto n, auto w) {
        constexpr int N = decltype(n)::value, W = decltype(w)::value;
        const int64_t blocks = W == 1 ? (rows + kWaves - 1) / kWaves : rows;
        hipLaunchKernelGGL((page_select_kernel<N, W>), dim3((unsigned)blocks), dim3(W == 1 ? kThreads : 64 * W), 0, st, a);
    };
    auto of_pages = [&](auto w) {
        constexpr int W = decltype(w)::value;
        const int64_t n = (pages + 64 * W - 1) / (64 * W);
        if (!need || n <= 2) return held(std::integral_constant<int, 2>{}, w);
        if (n <= 4) return held(std::integral_constant<int, 4>{}, w);
        if (W == 4 || n <= 8) return held(std::integral_constant<int, 8>{}, w);
        if constexpr (W != 4) {
            if (W == 16 || n <= 16) return held(std::integral_constant<int, 16>{}, w);
        }
        if constexpr (W == 1) held(std::integral_constant<int, 32>{}, w);
    };
    if (need && pages > kHeldPages)
        hipLaunchKernelGGL(page_select_wide_kernel, dim3((unsigned)rows), dim3(kWideThreads), 0, st, a);
    else if (need && pages > 64 * 32)
        of_pages(std::integral_constant<int, 16>{});
    else if (need && rows < 4096 && pages > 64)
        of_pages(std::integral_constant<int, 4>{});
    else
        of_pages(std::integral_constant<int, 1>{});
    return launch_status();
}

extern "C" size_t fkv_page_attend_selected_workspace(const fkv_page_desc* desc, const fkv_attend_desc* attend, int64_t n_selected)
{
    if (!attend_ok(desc, attend) || n_selected < 1 || n_selected > kMostListed) return 0;
    return listed_workspace(desc, attend, listed_shape(desc, attend, n_selected)).bytes;
}

extern "C" int fkv_page_attend_selected(const fkv_page_desc* desc, const fkv_attend_desc* attend, int64_t n_selected,
                                        const int32_t* selected, const uint8_t* k_codes, const uint8_t* v_codes,
                                        const float* scales, const void* q, const int32_t* tables, const int32_t* kv_len,
                                        const int32_t* q_start, const float* slopes, const int32_t* prefix, const int32_t* first,
                                        void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!attend_ok(desc, attend) || n_selected < 1 || n_selected > kMostListed) return FKV_ERR_INVALID_ARG;
    if (!k_codes || !v_codes || !scales || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(scales, 8))
        return FKV_ERR_INVALID_ARG;
    if (attend->n_req == 0 || attend->n_tokens == 0) return FKV_OK;
    if (!q || !out || !tables || !kv_len || !q_start || !selected || !aligned(q, 16) || !aligned(out, 16) || !aligned(tables, 4) ||
        !aligned(kv_len, 4) || !aligned(q_start, 4) || !aligned(selected, 4) || !aligned(slopes, 4) || !aligned(prefix, 4) ||
        !aligned(first, 4) || !aligned(lse, 4) || !aligned(workspace, 16))
        return FKV_ERR_INVALID_ARG;
    const ListedShape s = listed_shape(desc, attend, n_selected);
    const Workspace ws = listed_workspace(desc, attend, s);
    if (ws.bytes && (!workspace || workspace_bytes < ws.bytes)) return FKV_ERR_SCRATCH_TOO_SMALL;
    if (s.blocks > kMostBlocks / s.n_splits) return FKV_ERR_UNSUPPORTED;
    AttendArgs a = attend_args(desc, attend, k_codes, v_codes, scales, q, tables, kv_len, q_start, slopes, prefix, first, out, lse);
    a.listed = selected, a.n_listed = n_selected, a.searched = s.searched;
    a.part = (float*)workspace;
    a.stat = (float2*)((uint8_t*)workspace + ws.stat);
    a.n_splits = s.n_splits;
    const hipStream_t st = (hipStream_t)stream;
    const bool e4m3 = desc->format == FKV_PAGE_E4M3;
    auto of_width = [&](auto nc) {
        constexpr int NC = decltype(nc)::value;
        auto go = [&](auto kern, size_t shm) {
            hipLaunchKernelGGL(kern, dim3((unsigned)(s.blocks * s.n_splits)), dim3(s.waves == 1 ? kThreads : 64 * s.waves), shm, st, a);
        };
        const size_t shm = s.waves == 1 ? a.page % kTile ? 0 : (size_t)kWaves * kKeyBytes<NC>
                                        : (2 * s.waves * kFewRows + (size_t)s.waves * kFewRows * (a.d + 4)) * sizeof(float);
        auto of_form = [&](auto whole, auto plain) {
            constexpr bool WHOLE = decltype(whole)::value, PLAIN = decltype(plain)::value;
            auto of_waves = [&](auto w, auto u) {
                constexpr int W = decltype(w)::value, U = decltype(u)::value;
                e4m3 ? go(attend_listed_kernel<true, NC, W, WHOLE, PLAIN, U>, shm) : go(attend_listed_kernel<false, NC, W, WHOLE, PLAIN, U>, shm);
            };
            const std::integral_constant<int, 1> one;
            if (s.waves == 1) return a.group <= 4 ? of_waves(one, std::integral_constant<int, 4>{}) : of_waves(one, one);
            if constexpr (NC <= 2) {
                if (s.waves == 8) return of_waves(std::integral_constant<int, 8>{}, one);
            }
            of_waves(std::integral_constant<int, kWaves>{}, one);
        };
        const bool plain = a.softcap == 0.0f && !a.slopes;
        if (a.page % kTile == 0) plain ? of_form(std::true_type{}, std::true_type{}) : of_form(std::true_type{}, std::false_type{});
        else plain ? of_form(std::false_type{}, std::true_type{}) : of_form(std::false_type{}, std::false_type{});
    };
    if (a.d <= 64) of_width(std::integral_constant<int, 1>{});
    else if (a.d <= 128) of_width(std::integral_constant<int, 2>{});
    else of_width(std::integral_constant<int, 4>{});
    if (a.n_splits > 1) {
        const int64_t rows = (a.searched ? a.searched : a.n_req * a.max_new) * a.heads * a.group;   // (fewer than 256 items')
        const int64_t joins = s.join_blocks ? rows : (rows + kWaves - 1) / kWaves;
        hipLaunchKernelGGL(s.join_blocks ? attend_join_kernel<kWaves> : attend_join_kernel<1>, dim3((unsigned)joins), dim3(kThreads), 0, st, a);
    }
    return launch_status();
}
