// Decode over 4-bit caches (ST_MXFP4: E2M1 codes, one power of two per 32 dims of a token): the split kernel of
// st_decode.hip's scheme -- work units, partial results, the same merge -- and a form that finishes short caches in one launch.
//
// A token and KV head are D + D / 16 bytes, 136 at D = 128, against 4 D G flops for the G query rows that share them: bound by HBM, and only just.  A
// compute unit gets one 16-token page of a head every 220 cycles at 6 TB/s, and everything between the load and the matrix instruction has to fit
// into that.  Measured, 8 KV heads of 128 dims, the least of 40 launches (their mean is 3 to 16 % above): 64 sequences of up to 8K + 24K tokens, 4 rows a
// head: 217 us, 5.7 TB/s; 32 of 2K + up to 6K, 2 rows: 41 us, 4.9 TB/s; 64 of up to 8K + 16K, 8 tokens of 4 rows: 247 us, 3.7 TB/s, vector instructions 50 %
// and matrix instructions 27 % of the time.  The codes are laid out as the matrix instructions want them (st_kv_cache), one 16-byte load per lane, page and tensor:
//   K: lane (m = slot, g) holds 32 consecutive dims of its token -- one block, one scale.  The k-steps of the product take its four dwords in turn;
//      the query fragments use the same assignment of dims.
//   V: lane (m = dim % 16, g) holds slots 4 g .. + 3 of the D / 16 dims 16 j + m, which is what the score accumulator of lane group g holds
//      weights for: the weights go from one product into the other without an exchange.  A byte is dims d and d + 16 of ONE token, so one
//      conversion takes one scale.
// Codes become bf16 in registers, times their scale: exact (one bit of significand, powers of two).  (The matrix instruction that takes 4-bit codes
// and their scales as they are beside 8-bit ones, the queries as two of these, aligns the products of a step at some 12 bits of the largest: scores
// were off by 2^-12 of it, more than bf16 operands make.)
// Three workgroups per compute unit hide the loads: the next step's codes asked for a step ahead, in registers or in two sets in turn, cost a
// workgroup or registers that are not there, and were 0 to 10 % slower.
#include <algorithm>

#include "st_decode.h"

namespace st {

// the bytes of one step (64 tokens, four pages) that a lane holds
template <int D>
struct Codes {
    static constexpr int KW = D / 32, G = D / 32;       // dwords of K a lane holds per page; blocks of a row
    uint32_t k[4][KW], v[4][KW], vs[4][G];
    uint32_t ks[4];
};

template <int W>
__device__ __forceinline__ void load_words(uint32_t (&dst)[W], const uint8_t* base, uint32_t off) {
    const uint8_t* p = base + off;
    if constexpr (W == 4) {
        const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i] = x[i];
    } else {
        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
        dst[0] = x[0];
        dst[1] = x[1];
    }
}

// One cache of one (sequence, KV head) as a wave reads it: steps tok0, tok0 + stride * 64, ...; the page ids of its 16 steps at most are
// asked for before the cache's length is known (four lanes a step, ids clamped into the pool).
template <int D>
struct Pages4 {
    int my_page;
    const uint8_t *k_pool, *v_pool, *scales;
    __device__ __forceinline__ Pages4(const CacheView& cv, int b, int h, int lane, int tok0, int stride) {
        const int page = tok0 / kPage + 4 * stride * (lane >> 2) + (lane & 3);
        const int id = cv.page_table[int64_t(b) * cv.max_pages + min(page, cv.max_pages - 1)];
        my_page = min(max(id, 0), cv.n_pages - 1);
        k_pool = reinterpret_cast<const uint8_t*>(cv.k_pool) + h * (D * 8);
        v_pool = reinterpret_cast<const uint8_t*>(cv.v_pool) + h * (D * 8);
        scales = reinterpret_cast<const uint8_t*>(cv.k_scale) + h * D;
    }
    // step s of this cache, or of the other one where a wave walks both
    __device__ __forceinline__ void load(int s, int page, const uint8_t* kp, const uint8_t* vp, const uint8_t* sp, int n_kv_heads, Codes<D>& c) const {
        // (64 dims: two lane groups share a block of 32, half of it each.  A page's address stays scalar, beside an
        // unsigned 32-bit offset per lane, if the compiler sees the offset where it is used: without the empty statement it hoists its 64-bit form)
        uint32_t lane = threadIdx.x & 63u;
        asm volatile("" : "+v"(lane));
        const uint32_t n = lane & 15u, g = lane >> 4;
        const uint32_t k_off = D == 128 ? lane * 16u : (g >> 1) * 256u + n * 16u + (g & 1u) * 8u, v_off = lane * uint32_t(D / 8);
        const uint32_t ks_off = D == 128 ? lane : (g >> 1) * 16u + n, vs_off = uint32_t(D / 2) + g * uint32_t(D / 8);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = int64_t(__builtin_amdgcn_readlane(page, 4 * s + u)) * n_kv_heads;
            load_words(c.k[u], kp + at * (D * 8), k_off);
            load_words(c.v[u], vp + at * (D * 8), v_off);
            c.ks[u] = (sp + at * D)[ks_off];
            load_words(c.vs[u], sp + at * D, vs_off);
        }
    }
    __device__ __forceinline__ void load(int s, int n_kv_heads, Codes<D>& c) const { load(s, my_page, k_pool, v_pool, scales, n_kv_heads, c); }
};

// byte `i` of a scale word where the conversion looks for its exponent (it takes nothing else of the operand)
__device__ __forceinline__ float scale_of(uint32_t w, int i) { return __uint_as_float(i < 3 ? w << (23 - 8 * i) : w >> 1); }

// Running state of a wave: RB blocks of 16 columns, in base-2 exponent units; column n of block r in the lanes (n, g).
// Few query rows leave most of the 16 columns of a matrix instruction without a row of their own.  They hold the rows again -- COPIES times 16 / COPIES
// rows --, and each copy takes the softmax of its share of the step's four pages alone: the exponentials, which cost four times a multiplication, are
// not formed twice.  The copies share one reference exponent and their sums are added up at the end (fold_copies).
// Weights are the second product's in TWO bf16 parts, the rounded weight and, rounded, what that left: 2^-16 of a weight is lost at most, and the rows
// are as far from 64 bits as their own rounding takes them (1.63 to 1.66e-3 of their norm).  With the first part alone, 1.76 to 1.99e-3.  The second part costs up to eight
// rows nothing but some vector instructions: a copy has no weights of the other copies' pages, and there takes the second part of the row's weights
// from the copy that formed them.  More rows take twice the matrix instructions.  64 sequences of up to 8K + 16K tokens, 4, 8, 16 and 32 rows: 178, 181,
// 191 and 233 us with one part, 180, 183, 195 and 254 with two.
// The reference exponent of a column moves only when a score exceeds it, and then to 8 above that score, so that the exchange between lanes and the rescale
// of the accumulator are rare (32 rows 263 -> 254, 16 rows 197 -> 195): what the weights' parts leave is relative to the weight, whatever its size.  No weight is above
// 1, so that sums of large values stay where the values are.  The sum takes the weights as they are.
template <int D, int RB, int COPIES>
struct State4 {
    static constexpr int KS = D / 32, DB = D / 16, G = D / 32;
    static constexpr int ROWS = 16 / COPIES, OWN = 4 / COPIES;             // rows of a block; pages of a step that a column takes
    static constexpr float kRise = 8.f;
    static constexpr bool QUERIES_IN_LDS = RB > 1;                         // (one copy for the four waves, in fragment order [RB][KS][64 lanes])
    static constexpr bool SORT = COPIES == 1;                              // (9 rows or more: see the second product)
    bf16x8 q[QUERIES_IN_LDS ? 1 : KS];
    const bf16x8* s_q;
    f32x4 o[RB][DB];
    float m[RB], l[RB];
    __device__ __forceinline__ explicit State4(const bf16x8* lds) : s_q(lds) { clear(); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[r][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    static __device__ __forceinline__ int copy() { return (int(threadIdx.x) & 15) / ROWS; }
    // largest of the four lanes n, n + 16, n + 32, n + 48 of a column
    static __device__ __forceinline__ float column_max(float x) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
        return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    using By8 = std::integral_constant<int, 0x128>;                        // row_ror:8, row_ror:4
    using By4 = std::integral_constant<int, 0x124>;
    template <typename T, typename By>
    static __device__ __forceinline__ T from(T x, By) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), By::value, 0xf, 0xf, true));
    }
    // the bytes of a word's first n slots (n may be negative or more than four)
    static __device__ __forceinline__ uint32_t slots_below(int n) {
        uint32_t keep = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) keep |= i < n ? 0xffu << (8 * i) : 0u;
        return keep;
    }
    // 64 tokens from token `tok` of a cache of `len` visible tokens, of which this lane's column of block r sees [0, limit[r]) and every row
    // [0, limit_min).  EACH_LIMIT: see decode4_split_kernel.
    template <bool EACH_LIMIT>
    __device__ __forceinline__ void step(Codes<D>& c, int tok, int len, const int (&limit)[RB], int limit_min, float scale_log2) {
        const int lane = int(threadIdx.x) & 63, g = lane >> 4, mine = copy();
        f32x4 s[RB][4], t[RB][OWN];                                      // scores of page u: register i is slot 4 g + i
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int u = 0; u < 4; ++u) s[r][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            bf16x8 qf[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) qf[r] = QUERIES_IN_LDS ? s_q[(r * KS + j) * 64 + lane] : q[j];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                u32x4 kf;
#pragma unroll
                for (int i = 0; i < 4; ++i) kf[i] = fp4_pair(c.k[u][j], scale_of(c.ks[u], 0), i);
#pragma unroll
                for (int r = 0; r < RB; ++r) s[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), qf[r], s[r][u], 0, 0, 0);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) t[r][u % OWN][i] = u < OWN || mine == u / OWN ? s[r][u][i] : t[r][u % OWN][i];
        const int first = tok + 16 * OWN * mine + 4 * g;                 // token of t[.][0][0]; 16 further on for every other page
        if (tok + 64 > limit_min) {                                      // uniform: a step that reaches some row's limit
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                int left = limit[r] - first;
                if constexpr (RB > 1) asm volatile("" : "+v"(left));     // (a branch, not 32 selects in every step)
#pragma unroll
                for (int v = 0; v < OWN; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[r][v][i] = 16 * v + i < left ? t[r][v][i] : -INFINITY;
            }
        }
        uint32_t p[RB][OWN][SORT ? 2 : 4], rest[RB][OWN][SORT ? 2 : 4];  // both parts of the weights: pairs of slots, or one beside a 0 (rest: of the copy two
                                                                         // places, or one of two, further on)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int v = 0; v < OWN; ++v)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, t[r][v][i]);
            mx *= scale_log2;                                            // (which is positive)
            if (__any(mx > m[r])) {
                float top = column_max(mx);
                if constexpr (COPIES > 1) top = fmaxf(top, from(top, By8{}));
                if constexpr (COPIES == 4) top = fmaxf(top, from(top, By4{}));
                top = top > m[r] ? top + kRise : m[r];                   // (a column's own scores alone: no row's bits depend on another's)
                const float alpha = top > -INFINITY ? __builtin_amdgcn_exp2f(m[r] - top) : 1.f;
                m[r] = top;
                l[r] *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[r][db][i] *= alpha;
            }
            const float ref = m[r] > -INFINITY ? -m[r] : 0.f;            // (nothing seen so far, or NaN alone)
            float even = 0.f, odd = 0.f;
#pragma unroll
            for (int v = 0; v < OWN; ++v)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const float a = __builtin_amdgcn_exp2f(fmaf(t[r][v][i], scale_log2, ref)), b = __builtin_amdgcn_exp2f(fmaf(t[r][v][i + 1], scale_log2, ref));
                    even = v + i == 0 ? a : even + a;
                    odd = v + i == 0 ? b : odd + b;
                    if constexpr (SORT) {
                        const uint32_t w = pair_bf16(a, b);
                        p[r][v][i / 2] = w;
                        rest[r][v][i / 2] = pair_bf16(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
                    } else {
                        auto split = [&](float x, int e) {
                            p[r][v][e] = pair_bf16(x, 0.f);
                            rest[r][v][e] = from(pair_bf16(x - __uint_as_float(p[r][v][e] << 16), 0.f), By8{});
                        };
                        split(a, i);
                        split(b, i + 1);
                    }
                }
            l[r] += even + odd;
            asm volatile("" : "+v"(l[r]));                               // (the sums are formed here, not beside the second product: see decode4_split_kernel)
        }
        if (tok + 64 > len) {
            // slots past the visible length hold anything: their weights are 0, their scales must be finite
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t keep = slots_below(len - tok - 16 * u - 4 * g);
#pragma unroll
                for (int gg = 0; gg < G; ++gg) c.vs[u][gg] &= keep;
            }
        }
        // The second product.  A converted dword is one slot with dims 32 gg + m and 32 gg + 16 + m, two k-values of an operand whose columns are both
        // sets of dims.  Up to 8 rows: the weights go in twice, beside a 0 each, for the lower dims and for the upper ones -- twice the matrix
        // instructions, for which the pipe has the time.  More rows (SORT): the dwords of two slots are sorted into an operand of either
        // set, one more vector instruction per conversion for half the matrix instructions, of which the second parts of the weights take as many again.
        // One of its PIECES, into the accumulators sum(r, 0) of the lower and sum(r, 1) of the upper dims; scales(u): the scale word of page u.
        constexpr int PIECES = SORT ? 2 : 4;
        auto multiply = [&](int piece, int gg, auto scales, auto sum) {
            auto pair = [&](int u, int i) { return fp4_pair(c.v[u][gg], scale_of(scales(u), i), i); };
            auto add = [&](f32x4& x, const u32x4& v, const u32x4& w) { x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w), x, 0, 0, 0); };
            if constexpr (SORT) {
                u32x4 lo, hi;                                            // four slots of page 2 piece, four of the next
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t first = pair(2 * piece + (e >> 1), 2 * (e & 1)), second = pair(2 * piece + (e >> 1), 2 * (e & 1) + 1);
                    lo[e] = __builtin_amdgcn_perm(second, first, 0x05040100);
                    hi[e] = __builtin_amdgcn_perm(second, first, 0x07060302);
                }
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        const auto& x = part == 0 ? p[r] : rest[r];
                        const u32x4 w = {x[2 * piece][0], x[2 * piece][1], x[2 * piece + 1][0], x[2 * piece + 1][1]};
                        add(sum(r, 0), lo, w);
                        add(sum(r, 1), hi, w);
                    }
            } else {
                u32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = pair(piece, i);
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    u32x4 lo, hi;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lo[i] = mine == piece / OWN ? p[r][piece % OWN][i] : COPIES == 2 || (mine ^ 2) == piece / OWN ? rest[r][piece % OWN][i] : 0u;
                        hi[i] = lo[i] << 16;
                    }
                    add(sum(r, 0), v, lo);
                    add(sum(r, 1), v, hi);
                }
            }
        };
        if constexpr (!EACH_LIMIT) {
#pragma unroll
            for (int piece = 0; piece < PIECES; ++piece)
#pragma unroll
                for (int gg = 0; gg < G; ++gg) multiply(piece, gg, [&](int u) { return c.vs[u][gg]; }, [&](int r, int side) -> f32x4& { return o[r][2 * gg + side]; });
        } else {
            // for every limit in turn, with what lies past it cleared, into the columns that have this limit
            const bool alike = tok + 64 <= limit_min;
            for (int seen = alike ? len : limit_min; seen <= len; ++seen)
#pragma unroll
                for (int gg = 0; gg < G; ++gg) {
                    f32x4 x[RB][2];
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        x[r][0] = o[r][2 * gg];
                        x[r][1] = o[r][2 * gg + 1];
                    }
#pragma unroll
                    for (int piece = 0; piece < PIECES; ++piece)
                        multiply(piece, gg, [&](int u) { return c.vs[u][gg] & slots_below(seen - tok - 16 * u - 4 * g); }, [&](int r, int side) -> f32x4& { return x[r][side]; });
#pragma unroll
                    for (int r = 0; r < RB; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            o[r][2 * gg][i] = alike || limit[r] == seen ? x[r][0][i] : o[r][2 * gg][i];
                            o[r][2 * gg + 1][i] = alike || limit[r] == seen ? x[r][1][i] : o[r][2 * gg + 1][i];
                        }
                }
        }
    }
    // Whether any sum is infinite or undefined (0 times it is undefined)
    __device__ __forceinline__ bool past_finite() const {
        float none = 0.f;
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) none = fmaf(o[r][db][i], 0.f, none);
        return __any(none != 0.f);
    }
    // The four lanes of a column and the copies of a row merged, in a fixed order; afterwards every lane of a row holds its state.
    __device__ __forceinline__ void fold_copies() {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            l[r] += __shfl_xor(l[r], 16);
            l[r] += __shfl_xor(l[r], 32);
            if constexpr (COPIES > 1) {
                auto sum = [&](float x) {
                    x += from(x, By8{});
                    if constexpr (COPIES == 4) x += from(x, By4{});
                    return x;
                };
                l[r] = sum(l[r]);
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[r][db][i] = sum(o[r][db][i]);
            }
        }
    }
};

// Fragment j of the queries of (sequence b, KV head h), block r: row 16 r + n % (16 / COPIES) is token row / G, head row % G (rows past the end repeat
// the last one, never stored); dims D / 4 g + 8 j + e.  a.rope: rotated by the row's position, out of the table of the q_len positions.
template <int D, int COPIES>
__device__ __forceinline__ bf16x8 query_fragment(const DecodeArgs& a, int b, int h, int r, int j, const float2* s_rot) {
    const int lane = int(threadIdx.x) & 63, n = (lane & 15) % (16 / COPIES), d0 = (D / 4) * (lane >> 4) + 8 * j;
    const int row = min(16 * r + n, a.rows - 1), t = row / a.group;
    const uint16_t* qp = a.q + ((int64_t(b) * a.q_len + t) * a.n_q_heads + h * a.group + (row - t * a.group)) * D;
    bf16x8 x = *reinterpret_cast<const bf16x8*>(qp + d0);
    if (a.rope) {
        const bool upper = d0 >= D / 2;
        const int other0 = upper ? d0 - D / 2 : d0 + D / 2;
        const bf16x8 y = *reinterpret_cast<const bf16x8*>(qp + other0);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 cs = s_rot[t * (D / 2) + (upper ? other0 : d0) + e];
            const float own = float(x[e]), part = float(y[e]);
            x[e] = (__bf16)(upper ? own * cs.x + part * cs.y : own * cs.x - part * cs.y);
        }
    }
    return x;
}

// Row limits of a step over a cache: reasoning token j is seen by query token t where j <= len - q_len + t, the source slice by all
template <int RB, int COPIES>
__device__ __forceinline__ void row_limits(int (&limit)[RB], const DecodeArgs& a, bool is_src, int len) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int t = min(16 * r + (int(threadIdx.x) & 15) % (16 / COPIES), a.rows - 1) / a.group;
        limit[r] = is_src ? len : min(max(len - a.q_len + t + 1, 0), len);
    }
}

// Whether a block of the values of tokens first .. len - 1 (at most 31) may hold numbers that 0 times is not 0: a scale byte of 253 or more
template <int D>
__device__ __forceinline__ bool values_past_finite(const CacheView& cv, int b, int h, int first, int len) {
    constexpr int G = D / 32;
    bool found = false;
    for (int x = int(threadIdx.x) & 63; x < (len - first) * G; x += 64) {
        const int tok = first + x / G, slot = tok % kPage, id = cv.page_table[int64_t(b) * cv.max_pages + tok / kPage];
        const uint8_t* scales = reinterpret_cast<const uint8_t*>(cv.k_scale) + (int64_t(min(max(id, 0), cv.n_pages - 1)) * cv.n_kv_heads + h) * D;
        found = found || scales[D / 2 + ((slot >> 2) * G + x % G) * 4 + (slot & 3)] >= 253;
    }
    return __any(found);
}

// Three waves per SIMD leave 168 registers, and two blocks of rows at D = 128 take all of them.  A value that does not fit is one that each step begins
// with, and waits for in memory: with the weights kept for their sums until the second product there were four such values, the page ids among
// them, and a step of eight tokens of 64 sequences of up to 8K + 16K took 246 us, without them 229.
// SEVERAL tokens a step: the last of them are not seen by all rows, whose weights are 0 there, and 0 times a finite value is 0.  Where their blocks of values
// may hold others the product is formed limit by limit (EACH_LIMIT).  Here that is looked up before the first step, one more round trip (32 sequences of 2K +
// 2K tokens, 8 rows 28.5 us, so 30; 64 of up to 8K + 16K 182, 184): asked within the loop, or found in the sums at its end, with any state in common, the
// rare way costs the usual one registers (32 rows 250 us, with that 262 to 294; 8 rows 192).  One token a step is compiled without any of it.
template <int D, int RB, int COPIES, bool SEVERAL>
__global__ __launch_bounds__(64 * kSplitWaves, 3) void decode4_split_kernel(DecodeArgs a) {
    constexpr int DB = D / 16;
    // two blocks of rows: query fragments; behind them the (cos, sin) of the q_len query positions; after the loop: SplitLds
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const WaveStamp stamp(a);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nc = a.ncs + a.ncr;
    const unsigned bh = blockIdx.x / unsigned(nc);       // (sequence, KV head)
    const int c = unit_of(blockIdx.x, nc);
    const int h = int(bh % unsigned(a.n_kv_heads)), b = int(bh / unsigned(a.n_kv_heads));
    const bool is_src = c < a.ncs;
    const CacheView& cv = is_src ? a.src : a.rsn;
    const int unit0 = (is_src ? c : c - a.ncs) * a.chunk;
    const Pages4<D> pages(cv, b, h, lane, unit0 + 64 * wave, kSplitWaves);
    const int len = min(max(is_src ? a.src_len[b] : a.rsn_len[b], 0), cv.max_pages * kPage);
    if (unit0 >= len) return;
    const int n_steps = (min(len - unit0, a.chunk) - 64 * wave + 64 * kSplitWaves - 1) / (64 * kSplitWaves);
    const int limit_min = is_src ? len : min(max(len - a.q_len + 1, 0), len);
    const bool each_limit = SEVERAL && limit_min < min(len, unit0 + a.chunk) && values_past_finite<D>(cv, b, h, limit_min, len);
    using State = State4<D, RB, COPIES>;
    constexpr int KS = D / 32;
    bf16x8* s_q = reinterpret_cast<bf16x8*>(smem_raw);
    float2* s_rot = reinterpret_cast<float2*>(smem_raw + (State::QUERIES_IN_LDS ? RB * KS * 64 * sizeof(bf16x8) : 0));
    if (a.rope) {
        const int len_r = min(max(a.rsn_len[b], 0), a.rsn.max_pages * kPage);
        rope_table_to_lds<D>(s_rot, len_r - a.q_len, a.q_len, rope_frequency<D>(a.freq), 64 * kSplitWaves);
        lds_barrier();
    }
    if constexpr (State::QUERIES_IN_LDS) {
        for (int i = wave; i < RB * KS; i += kSplitWaves) s_q[i * 64 + lane] = query_fragment<D, COPIES>(a, b, h, i / KS, i % KS, s_rot);
        lds_barrier();
    }
    const int tok0 = unit0 + 64 * wave, n = lane & 15, g = lane >> 4;
    const int64_t slot = ((int64_t(b) * a.n_kv_heads + h) * nc + c) * a.rows;
    auto work = [&](auto each_limit, const Pages4<D>& pages, int len, int limit_min) {
        int limit[RB];
        row_limits<RB, COPIES>(limit, a, is_src, len);
        State st(s_q);
        if constexpr (!State::QUERIES_IN_LDS) {
#pragma unroll
            for (int j = 0; j < KS; ++j) st.q[j] = query_fragment<D, COPIES>(a, b, h, 0, j, s_rot);
        }
        for (int s = 0; s < n_steps; ++s) {
            Codes<D> codes;
            pages.load(s, a.n_kv_heads, codes);
            st.template step<decltype(each_limit)::value>(codes, tok0 + 64 * kSplitWaves * s, len, limit, limit_min, a.scale_log2);
        }
        st.fold_copies();
        // the waves' states meet in LDS, a block of rows at a time: with both at once (66 KB) a compute unit would hold two workgroups, not three
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            __syncthreads();                            // everybody is done with the queries and rotations, with the block before
            const int rows = min(a.rows - 16 * r, 16);
            const SplitLds<D> sm(smem_raw, rows);
            if (n < 16 / COPIES && n < rows) {
                // lane (n, g), block db, register i  <->  d = 16 db + 4 g + i
                float* po = sm.o + (wave * rows + n) * D;
#pragma unroll
                for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(po + 16 * db + 4 * g) = st.o[r][db];
                if (g == 0) {
                    sm.m[wave * rows + n] = st.m[r];
                    sm.l[wave * rows + n] = st.l[r];
                }
            }
            __syncthreads();
            merge_waves<D>(sm, rows, a, slot + 16 * r);
        }
    };
    // (the same for all waves)
    if (SEVERAL && each_limit) {
        int own_b = b, own_len = len, own_min = limit_min;
        asm volatile("" : "+s"(own_b), "+s"(own_len), "+s"(own_min));
        work(std::true_type{}, Pages4<D>(cv, own_b, h, lane, unit0 + 64 * wave, kSplitWaves), own_len, own_min);
    } else {
        work(std::false_type{}, pages, len, limit_min);
    }
}

// Short caches: a workgroup of eight waves takes all of a (sequence, KV head) and finishes its rows -- one launch, no partial results.  Steps are
// dealt out as in the bf16 kernel: reasoning steps from the first wave up, source steps from the last one down.
constexpr int kSmallWaves4 = 8;

template <int D, int COPIES, bool SEVERAL>
__global__ __launch_bounds__(64 * kSmallWaves4, 2) void decode4_small_kernel(DecodeArgs a, uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int DB = D / 16, W = kSmallWaves4;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    float* sm_o = reinterpret_cast<float*>(smem_raw);
    float2* sm_ml = reinterpret_cast<float2*>(sm_o + W * a.rows * D);
    float2* sm_rot = sm_ml + W * a.rows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = int(blockIdx.x % unsigned(a.n_kv_heads)), b = int(blockIdx.x / unsigned(a.n_kv_heads));
    const Pages4<D> first_s(a.src, b, h, lane, 64 * (W - 1 - wave), W), first_r(a.rsn, b, h, lane, 64 * wave, W);
    const int len_s = min(max(a.src_len[b], 0), a.src.max_pages * kPage), len_r = min(max(a.rsn_len[b], 0), a.rsn.max_pages * kPage);
    const int steps_s = (len_s - 64 * (W - 1 - wave) + 64 * W - 1) / (64 * W), steps_r = (len_r - 64 * wave + 64 * W - 1) / (64 * W);
    const int limit_min = min(max(len_r - a.q_len + 1, 0), len_r);
    if (a.rope) {
        rope_table_to_lds<D>(sm_rot, len_r - a.q_len, a.q_len, rope_frequency<D>(a.freq), 64 * W);
        lds_barrier();
    }
    State4<D, 1, COPIES> st(nullptr);
    auto walk = [&](auto each_limit, const Pages4<D>& pages_s, const Pages4<D>& pages_r, int b, int len_s, int len_r, int limit_min) {
        int limit_s[1], limit_r[1];
        row_limits<1, COPIES>(limit_s, a, true, len_s);
        row_limits<1, COPIES>(limit_r, a, false, len_r);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) st.q[j] = query_fragment<D, COPIES>(a, b, h, 0, j, sm_rot);
        for (int x = 0; x < steps_r + steps_s; ++x) {
            const bool r = x < steps_r;
            const int s = r ? x : x - steps_r;
            Codes<D> codes;
            pages_r.load(s, r ? pages_r.my_page : pages_s.my_page, r ? pages_r.k_pool : pages_s.k_pool, r ? pages_r.v_pool : pages_s.v_pool,
                         r ? pages_r.scales : pages_s.scales, a.n_kv_heads, codes);
            const int limit[1] = {r ? limit_r[0] : limit_s[0]};
            st.template step<decltype(each_limit)::value>(codes, 64 * ((r ? wave : W - 1 - wave) + W * s), r ? len_r : len_s, limit, r ? limit_min : len_s, a.scale_log2);
        }
    };
    walk(std::false_type{}, first_s, first_r, b, len_s, len_r, limit_min);
    // (SEVERAL, EACH_LIMIT: see decode4_split_kernel.  Here a wave finds in its sums, at no cost, that it has to walk again: looked up before, 0.6 us of 9.)
    if (SEVERAL && __builtin_expect(limit_min < len_r && 64 * (wave + W * (steps_r - 1)) + 64 > limit_min && st.past_finite(), 0)) {
        int own_b = b, own_s = len_s, own_r = len_r, own_min = limit_min;
        asm volatile("" : "+s"(own_b), "+s"(own_s), "+s"(own_r), "+s"(own_min));
        st.clear();
        walk(std::true_type{}, Pages4<D>(a.src, own_b, h, lane, 64 * (W - 1 - wave), W), Pages4<D>(a.rsn, own_b, h, lane, 64 * wave, W), own_b, own_s, own_r, own_min);
    }
    st.fold_copies();
    const int n = lane & 15, g = lane >> 4;
    if (n < 16 / COPIES && n < a.rows) {
        float* po = sm_o + (wave * a.rows + n) * D;
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(po + 16 * db + 4 * g) = st.o[0][db];
        if (g == 0) sm_ml[wave * a.rows + n] = float2{st.m[0], st.l[0]};
    }
    __syncthreads();
    merge_and_store<D, W, W>(sm_o, sm_ml, a, b, h, out, lse);
}

template <typename Kernel>
static st_status allow_lds(Kernel kernel, size_t bytes) {
    if (bytes > 64 * 1024)                              // beyond the default limit
        ST_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(bytes)));
    return ST_OK;
}

st_status launch_decode4(const DecodeArgs& a, int head_dim, int64_t units, hipStream_t s) {
    const size_t loop = (a.rows > 16 ? size_t(2) * (head_dim / 32) * 64 * 16 : 0) + size_t(a.q_len) * (head_dim / 2) * sizeof(float2);
    const size_t smem = std::max(loop, split_lds_bytes(std::min(a.rows, 16), head_dim));
    auto go = [&](auto kernel) -> st_status {
        const st_status r = allow_lds(kernel, smem);
        if (r == ST_OK) hipLaunchKernelGGL(kernel, dim3((unsigned)units), dim3(64 * kSplitWaves), smem, s, a);
        return r;
    };
    auto pick = [&](auto several) -> st_status {
        constexpr bool S = decltype(several)::value;
        if (a.rows <= 4) return head_dim == 64 ? go(decode4_split_kernel<64, 1, 4, S>) : go(decode4_split_kernel<128, 1, 4, S>);
        if (a.rows <= 8) return head_dim == 64 ? go(decode4_split_kernel<64, 1, 2, S>) : go(decode4_split_kernel<128, 1, 2, S>);
        return head_dim == 64 ? go(decode4_split_kernel<64, 1, 1, S>) : go(decode4_split_kernel<128, 1, 1, S>);
    };
    if (a.rows <= 16) return a.q_len == 1 ? pick(std::false_type{}) : pick(std::true_type{});
    return head_dim == 64 ? go(decode4_split_kernel<64, 2, 1, true>) : go(decode4_split_kernel<128, 2, 1, true>);
}

st_status launch_decode4_small(const DecodeArgs& a, int head_dim, uint16_t* out, float* lse, hipStream_t s) {
    const size_t smem = (size_t(kSmallWaves4) * a.rows * (head_dim + 2) + size_t(a.q_len) * head_dim) * sizeof(float);
    auto go = [&](auto kernel) -> st_status {
        const st_status r = allow_lds(kernel, smem);
        if (r == ST_OK) hipLaunchKernelGGL(kernel, dim3((unsigned)(a.batch * a.n_kv_heads)), dim3(64 * kSmallWaves4), smem, s, a, out, lse);
        return r;
    };
    auto pick = [&](auto several) -> st_status {
        constexpr bool S = decltype(several)::value;
        if (a.rows <= 4) return head_dim == 64 ? go(decode4_small_kernel<64, 4, S>) : go(decode4_small_kernel<128, 4, S>);
        if (a.rows <= 8) return head_dim == 64 ? go(decode4_small_kernel<64, 2, S>) : go(decode4_small_kernel<128, 2, S>);
        return head_dim == 64 ? go(decode4_small_kernel<64, 1, S>) : go(decode4_small_kernel<128, 1, S>);
    };
    return a.q_len == 1 ? pick(std::false_type{}) : pick(std::true_type{});
}

}  // namespace st
