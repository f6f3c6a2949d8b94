// Rows of paged caches in any of the storage formats: new tokens' keys normalised, rotated, coded and stored in one launch
// (st_kv_append_norm_rope; 4-bit caches also in st_kv_append and st_kv_append_rope), and stored rows read back (st_kv_read).
//
// Pure data movement, bound by HBM where there is much of it and by the chain of memory round trips where there is a
// token per sequence.  A workgroup takes ONE page of a sequence that the call touches and some KV heads of it (all of them where there are pages
// enough), so that the angles of the page's tokens are evaluated once for all heads.  A row lies in D / 8 neighbouring lanes, eight
// dims each, as in the normalising kernels.
//
// Keys are normalised and rotated in 64 bits and rounded to bf16 once; codes are formed from those bf16 rows.  64 bits, because a code is
// as wide as a sixth of its block's largest value: 32 bits would put a few keys of every million on the other side of the line between two codes,
// and the same row would not always be stored alike.  Nearly every row's codes are the same at both ends of the interval that 32-bit arithmetic
// leaves, though, and those rows are done with it (quick_key).
//
// Measured, 4 bits, 8 heads of 128 dims, calls repeated in a captured graph.  16 documents, 45,630 tokens (187 MB of rows, 50 of codes): stored in 71 us, the rows of a cache
// without norm and rotation in 56, read back in 59, one after the other in 120; nothing between the loads and the stores but the codes, loads
// two to eight passes ahead, rows in the order in which they lie: each within 3 % of that, so it is
// memory (at the rate of a large copy 45).  32,768 tokens of rows into 16 bits 73 us, 8 bits 66, 4 bits 54; out again 60, 50 and 43.  64 sentences of up to 190 tokens: 18 and
// 9 us; a token for each of 64: 5.3 and 3.3.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "st_cache.h"
#include "st_norm.h"

namespace st {

struct RowsArgs {
    CacheView cache;
    const uint16_t* k_new;       // [batch][max_new] tokens of [n_kv_heads][D]; elements from a token to the next: k_stride, v_stride
    const uint16_t* v_new;
    int64_t k_stride, v_stride;
    const int32_t* start_len;    // [batch] index of the first new token, or null: appended_len
    const int32_t* n_new;
    int max_new, touched;        // tokens per sequence; pages per sequence that the call may touch
    int heads, head_groups;      // KV heads of a workgroup, workgroups per page
    const uint16_t* k_weight;
    double eps;
    int rotate, write_len;       // write_len: the workgroup of a sequence's first page writes the new length
    RopeTable rope;
};
struct PagesArgs : RowsArgs {
    double2 step[64];            // (cos, sin) of the pairs' angles per token
};

// 64 bits rounded to bf16 in ONE rounding: to 32 bits with the last bit set if anything was lost, then to nearest even
__device__ __forceinline__ uint32_t f64_to_bf16_bits(double x) {
    const float f = float(x);
    uint32_t u = __float_as_uint(f);
    if (double(f) != x) {
        if (fabs(double(f)) > fabs(x)) u -= 1;
        u |= 1u;
    }
    return f32_to_bf16_bits(__uint_as_float(u));
}
// Eight at once.  By way of 32 bits, rounded to nearest, the result is the same unless the 32-bit value lies exactly between two bf16 values (its
// lower half is 0x8000): a lane that has such a value, one in some thousands, takes the long way with all of them.
__device__ __forceinline__ u32x4 f64x8_to_bf16(const double (&x)[8]) {
    uint32_t f[8];
    u32x4 out;
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 between = {0xffffu, 0xffffu};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __float_as_uint(float(x[i]));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x2 r;
        r[0] = (__bf16)__uint_as_float(f[2 * i]);
        r[1] = (__bf16)__uint_as_float(f[2 * i + 1]);
        out[i] = __builtin_bit_cast(uint32_t, r);
        const uint32_t lower = __builtin_amdgcn_perm(f[2 * i + 1], f[2 * i], 0x05040100) ^ 0x80008000u;
        between = __builtin_elementwise_min(between, __builtin_bit_cast(u16x2, lower));
    }
    if (between[0] == 0 || between[1] == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = f64_to_bf16_bits(x[2 * i]) | (f64_to_bf16_bits(x[2 * i + 1]) << 16);
    return out;
}
// x^(-1/2) in 64 bits: the instruction's estimate and Newton's iteration (each squares the error)
__device__ __forceinline__ double inverse_root(double x) {
    double y = __builtin_amdgcn_rsq(x);
    const double h = 0.5 * x;
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(y, fma(-h * y, y, 0.5), y);
    return y;
}

constexpr int kScaleExpLeast = -100;             // of 8-bit rows and 4-bit blocks alike

// Largest magnitude (as bf16 bits, non-finite above all, or left out) of a lane's eight values, over LANES neighbouring lanes
template <int LANES, bool FINITE = false>
__device__ __forceinline__ uint32_t row_top(const u32x4& x) {
    uint32_t top = 0;
    auto magnitude = [](uint32_t m) { return FINITE && m >= 0x7f80u ? 0u : m; };
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(magnitude(x[i] & 0x7fffu), magnitude((x[i] >> 16) & 0x7fffu)));
    auto fold = [&](auto ctrl) { top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), decltype(ctrl)::value, 0xf, 0xf, true))); };
    fold(std::integral_constant<int, 0xb1>{});
    fold(std::integral_constant<int, 0x4e>{});
    if constexpr (LANES >= 8) fold(std::integral_constant<int, 0x141>{});
    if constexpr (LANES >= 16) fold(std::integral_constant<int, 0x140>{});
    return top;
}
// The smallest k from -100 on with (bf16 bits) top <= m 2^(e + k), m = 1 + m128 / 128; 0 for top = 0
__device__ __forceinline__ int scale_exponent(uint32_t top, int m128, int e) {
    const int k = max(int((top + uint32_t(127 - m128)) >> 7) - 127 - e, kScaleExpLeast);         // (a significand above m carries)
    return top == 0 ? 0 : k;
}

// Storage formats.  encode: a lane's eight values (bf16, of dims 8 c ..) as the format's codes, with the scale's exponent; put_*: to the token's place
// in a page of one head.  PIECE: bytes of the eight.
template <int FMT, int D>
struct Store;

template <int D>
struct Store<ST_BF16, D> {
    static constexpr int PIECE = 16;
    using Code = u32x4;
    static __device__ __forceinline__ Code encode(const u32x4& x) { return x; }
    static __device__ __forceinline__ void put_scale(const CacheView&, int64_t, int, int, bool, const Code&) {}
    static __device__ __forceinline__ void put_key(uint8_t* page, int slot, int c, const Code& p) { *reinterpret_cast<u32x4*>(page + (c * kPage + slot) * 16) = p; }
    static __device__ __forceinline__ void put_value(uint8_t* page, int slot, int c, const Code& p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) *reinterpret_cast<uint16_t*>(page + ((8 * c + e) * kPage + slot) * 2) = uint16_t(p[e / 2] >> (16 * (e & 1)));
    }
};

template <int D>
struct Store<ST_FP8_E4M3, D> {
    static constexpr int PIECE = 8;
    struct Code {
        uint32_t w[2];
        int k;
    };
    static __device__ __forceinline__ bool same(const Code& a, const Code& b) { return a.w[0] == b.w[0] && a.w[1] == b.w[1] && a.k == b.k; }
    static __device__ __forceinline__ Code encode(const u32x4& x) {
        // (448 = 1.75 * 2^8; an infinite or undefined element has a code of its own, the scale is the others')
        Code r;
        r.k = scale_exponent(row_top<D / 8, true>(x), 96, 8);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float f[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f[2 * i] = ldexpf(__uint_as_float(x[2 * u + i] << 16), -r.k);
                f[2 * i + 1] = ldexpf(__uint_as_float(x[2 * u + i] & 0xffff0000u), -r.k);
            }
            r.w[u] = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0u, false);
            r.w[u] = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], r.w[u], true);
        }
        return r;
    }
    static __device__ __forceinline__ void put_scale(const CacheView& cv, int64_t page_head, int slot, int c, bool value, const Code& p) {
        if (c == 0) (value ? cv.v_scale : cv.k_scale)[page_head * kPage + slot] = ldexpf(1.f, p.k);
    }
    static __device__ __forceinline__ void put_key(uint8_t* page, int slot, int c, const Code& p) {
        *reinterpret_cast<u32x2*>(page + ((c >> 1) * kPage + slot) * 16 + 8 * (c & 1)) = u32x2{p.w[0], p.w[1]};
    }
    static __device__ __forceinline__ void put_value(uint8_t* page, int slot, int c, const Code& p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) page[(8 * c + e) * kPage + slot] = uint8_t(p.w[e / 4] >> (8 * (e & 3)));
    }
};

// 4 bits: see st_kv_cache.  A value byte holds dims d and d + 16 of one token, so that no byte is shared between tokens: the lanes of dims
// 8 c and 8 (c ^ 2) exchange codes, and each writes four of the eight bytes that the two have in common.
template <int D>
struct Store<ST_MXFP4, D> {
    static constexpr int PIECE = 4;
    struct Code {
        uint32_t w, scale;       // scale: the E8M0 byte
    };
    static __device__ __forceinline__ bool same(const Code& a, const Code& b) { return a.w == b.w && a.scale == b.scale; }
    static __device__ __forceinline__ Code encode(const u32x4& x) {
        const uint32_t top = row_top<4>(x);                  // a block of 32 dims: four lanes
        const bool bad = top >= 0x7f80u;
        const uint32_t biased = uint32_t(scale_exponent(top, 64, 2) + 127);                      // 6 = 1.5 * 2^2
        const float scale = __uint_as_float(biased << 23);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[1] << 16), __uint_as_float(x[1] & 0xffff0000u), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[2] << 16), __uint_as_float(x[2] & 0xffff0000u), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[3] << 16), __uint_as_float(x[3] & 0xffff0000u), scale, 3);
        return Code{bad ? 0u : w, bad ? 255u : biased};
    }
    static __device__ __forceinline__ void put_scale(const CacheView& cv, int64_t page_head, int slot, int c, bool value, const Code& p) {
        if ((c & 3) != 0) return;
        uint8_t* scales = reinterpret_cast<uint8_t*>(cv.k_scale) + page_head * D;
        scales[value ? D / 2 + ((slot >> 2) * (D / 32) + (c >> 2)) * 4 + (slot & 3) : (c >> 2) * kPage + slot] = uint8_t(p.scale);
    }
    static __device__ __forceinline__ void put_key(uint8_t* page, int slot, int c, const Code& p) {
        *reinterpret_cast<uint32_t*>(page + ((c >> 2) * kPage + slot) * 16 + 4 * (c & 3)) = p.w;
    }
    static __device__ __forceinline__ void put_value(uint8_t* page, int slot, int c, const Code& p) {
        const uint32_t mine = p.w, other = uint32_t(__builtin_amdgcn_update_dpp(0, int(mine), 0x4e, 0xf, 0xf, true));       // lane c ^ 2
        const bool high = (c & 2) != 0;                     // this lane holds the dims 16 further on
        // this lane's four of the eight: dims 8 (c % 2) + first .. + 3 within sixteen; their codes as the nibbles of 16 bits
        const int first = high ? 4 : 0;
        const uint32_t lo = ((high ? other : mine) >> (4 * first)) & 0xffffu, hi = ((high ? mine : other) >> (4 * first)) & 0xffffu;
        uint8_t* dst = page + ((slot >> 2) * 16 + 8 * (c & 1) + first) * (D / 8) + (c >> 2) * 4 + (slot & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i * (D / 8)] = uint8_t(((lo >> (4 * i)) & 15u) | (((hi >> (4 * i)) & 15u) << 4));
    }
};

// A key row's eight dims in a lane, normalised and rotated in 64 bits; angles: (cos, sin) times a of the token's pairs
template <int D>
__device__ __forceinline__ u32x4 exact_key(const u32x4& raw, const RowsArgs& a, const u32x4& w_raw, const double2* angles) {
    constexpr int L = D / 8;
    double x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = double(__uint_as_float(raw[i] << 16));
        x[2 * i + 1] = double(__uint_as_float(raw[i] & 0xffff0000u));
    }
    if (a.k_weight) {
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fma(x[i], x[i], ss);
        const double r = inverse_root(fma(row_sum<L>(ss), 1.0 / D, a.eps));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] *= r * double(__uint_as_float(w_raw[i] << 16));
            x[2 * i + 1] *= r * double(__uint_as_float(w_raw[i] & 0xffff0000u));
        }
    }
    if (a.rotate) {
        const RowTurn turn(a.rope, int(threadIdx.x) % L);
        if (a.rope.interleaved) {
            if (turn.turned) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double2 r = angles[turn.at + i];
                    const double lo = x[2 * i], hi = x[2 * i + 1];
                    x[2 * i] = lo * r.x - hi * r.y;
                    x[2 * i + 1] = hi * r.x + lo * r.y;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double other = __shfl(x[i], turn.partner);
                if (turn.turned) {
                    const double2 r = angles[turn.at + i];
                    x[i] = x[i] * r.x + other * (turn.high ? r.y : -r.y);
                }
            }
        }
    }
    return f64x8_to_bf16(x);
}

// Where a lane finds the angles of its dims in 32 bits.  Dims past the rotated ones have angles of their own, (1, 0), behind the table, so that
// no lane has to be told apart; the sines are there with either sign, for the lower and for the upper dims of their pairs.
struct QuickTurn {
    int cos_at, cos_step, sin_at, sin_step;      // from the tables' beginnings; from a token to the next
    float unit;                                  // what a rounding is of (|n_i| + |n_j|), see quick_key
};

// The same in 32 bits: bf16 rows (lo, hi) between whose MAGNITUDES the row in 64 bits lies, value by value; false if the row's size is not of 32 bits.
// By magnitude, because a block's scale goes by its largest: k(lo) <= k <= k(hi), and where the scales are equal the codes are as monotone, so equal codes
// at both ends are the row's.  (By value, the largest of either sign next to one line between two scales would put BOTH ends past it.)  A value that may be
// of either sign has codes of either sign at its ends, zeros too.
// Roundings, in units of u = 2^-24, of y = r (c n_i + s n_j) with n = x w, which is exact: c and s 1 each, the product and the sum 2, r, which is formed
// in 64 bits, and the last product 1 each: 5 a r (|n_i| + |n_j|) in all, taken as 6.  (The mean in 32 bits as well, 13: twice as many rows without
// a single bf16 row between their ends.)
template <int D>
__device__ __forceinline__ bool quick_key(const u32x4& raw, const RowsArgs& a, const u32x4& w_raw, const QuickTurn& turn, int partner, const float* cos, const float* sin,
                                          u32x4& lo, u32x4& hi) {
    constexpr int L = D / 8;
    float x[8], size[8], r = 1.f;
    bool sure = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(raw[i] << 16);
        x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
    if (a.k_weight) {
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fma(double(x[i]), double(x[i]), ss);
        const double mean = fma(row_sum<L>(ss), 1.0 / D, a.eps);
        sure = mean > 0x1p-60 && mean < 0x1p80;
        r = float(inverse_root(mean));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] *= __uint_as_float(w_raw[i] << 16);
            x[2 * i + 1] *= __uint_as_float(w_raw[i] & 0xffff0000u);
        }
    }
    if (a.rotate && a.rope.interleaved) {
        const f32x4 c = *reinterpret_cast<const f32x4*>(cos), s = *reinterpret_cast<const f32x4*>(sin);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = x[2 * i], q = x[2 * i + 1];
            size[2 * i] = size[2 * i + 1] = fabsf(p) + fabsf(q);
            x[2 * i] = fmaf(p, c[i], -(q * s[i]));
            x[2 * i + 1] = fmaf(q, c[i], p * s[i]);
        }
    } else if (a.rotate) {
        float other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl(x[i], partner);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const f32x4 c = *reinterpret_cast<const f32x4*>(cos + 4 * u), s = *reinterpret_cast<const f32x4*>(sin + 4 * u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 4 * u + i;
                size[e] = fabsf(x[e]) + fabsf(other[e]);
                x[e] = fmaf(x[e], c[i], other[e] * s[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) size[i] = fabsf(x[i]);
    }
    if (!a.k_weight) {
        // (nothing has made these sizes ordinary: past 2^100 a product or the interval's ends might pass 2^128; undefined: not below it)
#pragma unroll
        for (int i = 0; i < 8; ++i) sure = sure && size[i] < 0x1p100f;
    }
    const float unit = turn.unit * r;
    bf16x8 l, h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float err = copysignf(unit * size[i], x[i]);
        l[i] = (__bf16)fmaf(x[i], r, -err);
        h[i] = (__bf16)fmaf(x[i], r, err);
    }
    lo = __builtin_bit_cast(u32x4, l);
    hi = __builtin_bit_cast(u32x4, h);
    return sure;
}

constexpr int kRowsThreads = 256;

// Args: PagesArgs; RowsArgs for a single token per sequence, which needs no angles but its own: a kilobyte of arguments less to hand over (the call
// 4.7 -> 4.2 us on the host) and no whole pages to tell apart (a token for each of 64 sequences 5.4 -> 4.8).
template <int FMT, int D, typename Args>
__global__ __launch_bounds__(kRowsThreads) void append_rows_kernel(Args a) {
    using S = Store<FMT, D>;
    constexpr bool ONE = std::is_same_v<Args, RowsArgs>;
    constexpr int L = D / 8, RP = kRowsThreads / L, HEADS = RP / kPage;      // rows, whole pages of a head per pass
    constexpr int IMAGE = D * kPage * S::PIECE / 8;                          // bytes of a page of one head
    // In LDS the values of eight dims lie 16 bytes further on per lane: 128 or 256 bytes apart, all lanes of a row would write into two banks, or
    // one.  (4 bits: a lane's bytes are spread as they are.)
    constexpr int GAP = FMT == ST_MXFP4 ? 0 : 16, RUN = IMAGE / L, PADDED = IMAGE + GAP * L;
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr bool CODED = FMT != ST_BF16;
    // (cos, sin) times a of sixteen tokens, [16][rot / 2]; in 32 bits the cosines, the sines with either sign, [16][rot], and the angles of dims past
    // the rotated ones (not for bf16 rows, which are all formed in 64 bits: a fifth of the waves would be, behind the others' longer chain -- 64 sentences
    // of 64 tokens 15 us, so 19)
    const int half = a.rope.rot / 2, angles = a.rotate ? kPage * half : 0;
    double2* table = reinterpret_cast<double2*>(smem);
    float *s_cos = reinterpret_cast<float*>(table + angles), *s_sin = s_cos + angles, *s_none = s_sin + 2 * angles;
    uint8_t* image = reinterpret_cast<uint8_t*>(CODED && a.rotate ? s_none + 16 : s_cos);                 // [2][HEADS][PADDED]
    const int group = int(blockIdx.x) % a.head_groups, pi = (int(blockIdx.x) / a.head_groups) % a.touched, b = int(blockIdx.x) / (a.head_groups * a.touched);
    const int capacity = a.cache.max_pages * kPage;
    const int h0 = group * a.heads, n_heads = min(a.heads, a.cache.n_kv_heads - h0);
    const int c = int(threadIdx.x) % L, row = int(threadIdx.x) / L;
    // one token per sequence: its rows do not depend on the lengths, and are asked for before them
    u32x4 k_next = {0u, 0u, 0u, 0u}, v_next = {0u, 0u, 0u, 0u};
    if (ONE && row < n_heads) {
        k_next = *reinterpret_cast<const u32x4*>(a.k_new + b * a.k_stride + (h0 + row) * D + 8 * c);
        v_next = *reinterpret_cast<const u32x4*>(a.v_new + b * a.v_stride + (h0 + row) * D + 8 * c);
    }
    u32x4 w_raw = {0u, 0u, 0u, 0u};
    if (a.k_weight) w_raw = *reinterpret_cast<const u32x4*>(a.k_weight + 8 * c);
    const int start = min(max(a.start_len ? a.start_len[b] : a.cache.appended_len[b], 0), capacity);
    int n = a.n_new ? min(max(a.n_new[b], 0), a.max_new) : a.max_new;
    n = min(n, capacity - start);                                            // tokens past the page table are dropped
    if (a.write_len) {
        // (a length that this launch also reads is read by this workgroup alone)
        __syncthreads();
        if (pi == 0 && group == 0 && threadIdx.x == 0) a.cache.appended_len[b] = start + n;
    }
    const int page = start / kPage + pi;
    const int lo = max(start, page * kPage), hi = min(start + n, (page + 1) * kPage);
    if (lo >= hi) return;
    const int id = a.cache.page_table[int64_t(b) * a.cache.max_pages + page];              // (looked at behind the angles)
    const int slot_lo = lo - page * kPage, cnt = ONE ? 1 : hi - lo;
    const int64_t tok0 = int64_t(b) * a.max_new + (lo - start);
    if (a.rotate) {
        // four consecutive tokens of a pair per thread: one evaluation at the first (a token's index is its position id), then turned on by the pair's
        // angle per token
        for (int w = int(threadIdx.x); w < (cnt + 3) / 4 * half; w += kRowsThreads) {
            const int t0 = w / half, i = w - t0 * half;
            const double rev = double(lo + 4 * t0) * a.rope.f[i] * 0.15915494309189535;          // angle / 2 pi
            double2 r;
            sincospi(2.0 * (rev - rint(rev)), &r.y, &r.x);
            r.x *= a.rope.a;
            r.y *= a.rope.a;
            auto keep = [&](int t) {
                table[t * half + i] = r;
                if constexpr (CODED) {
                    s_cos[t * half + i] = float(r.x);
                    s_sin[t * 2 * half + i] = -float(r.y);
                    s_sin[t * 2 * half + half + i] = float(r.y);
                }
            };
            if constexpr (ONE) {
                keep(0);
            } else {
                const double2 step = a.step[i];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    keep(4 * t0 + t);                                // (the table holds sixteen tokens)
                    r = double2{r.x * step.x - r.y * step.y, r.y * step.x + r.x * step.y};
                }
            }
        }
        if (CODED && threadIdx.x < 16) s_none[threadIdx.x] = threadIdx.x < 8 ? 1.f : 0.f;
        __syncthreads();
    }
    if (id < 0 || id >= a.cache.n_pages) return;                             // never write outside the pool
    QuickTurn quick = {0, 0, 0, 0, 6.f / 16777216.f};
    int partner = int(threadIdx.x) & 63;
    // (sizes at which nothing overflows in 32 bits, and what is lost under 2^-126 is under 2^-116 in the key)
    bool usual = true;
    if (a.rotate) {
        const RowTurn turn(a.rope, c);
        partner = turn.partner;
        quick = turn.turned ? QuickTurn{turn.at, half, a.rope.interleaved ? half + turn.at : 8 * c, 2 * half, quick.unit * float(a.rope.a)}
                            : QuickTurn{int(s_none - s_cos), 0, int(s_none + 8 - s_sin), 0, quick.unit};
        usual = a.rope.a < 0x1p20 && a.rope.a > 0x1p-20;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) usual = usual && (w_raw[i] & 0x7fffu) <= 0x4980u && ((w_raw[i] >> 16) & 0x7fffu) <= 0x4980u;
    auto load = [&](const uint16_t* src, int64_t stride, int t, int h) { return *reinterpret_cast<const u32x4*>(src + (tok0 + t) * stride + (h0 + h) * D + 8 * c); };
    auto page_of = [&](uint16_t* pool, int h) { return reinterpret_cast<uint8_t*>(pool) + (int64_t(id) * a.cache.n_kv_heads + h0 + h) * IMAGE; };
    auto key = [&](const u32x4& raw, int t) -> typename S::Code {
        if (!a.k_weight && !a.rotate) return S::encode(raw);
        if constexpr (CODED) {
            // (the same bf16 row at both ends in four waves of five, the same codes in nearly all others)
            u32x4 x_lo, x_hi;
            const bool sure = quick_key<D>(raw, a, w_raw, quick, partner, s_cos + quick.cos_at + t * quick.cos_step, s_sin + quick.sin_at + t * quick.sin_step, x_lo, x_hi) && usual;
            const uint32_t apart = (x_lo[0] ^ x_hi[0]) | (x_lo[1] ^ x_hi[1]) | (x_lo[2] ^ x_hi[2]) | (x_lo[3] ^ x_hi[3]);
            const typename S::Code code = S::encode(x_lo);
            if (!__any(!sure || apart != 0)) return code;
            if (!__any(!sure || !S::same(code, S::encode(x_hi)))) return code;
        }
        return S::encode(exact_key<D>(raw, a, w_raw, table + t * half));
    };
    auto put = [&](const typename S::Code& code, bool value, uint8_t* page, int64_t page_head, int slot) {
        S::put_scale(a.cache, page_head, slot, c, value, code);
        if (value) S::put_value(page, slot, c, code);
        else S::put_key(page, slot, c, code);
    };

    if (ONE || cnt < kPage) {
        // part of a page: rows (head, token) in turn, straight to their places
        for (int r = row; r < cnt * n_heads; r += RP) {
            const int h = r / cnt, t = r - h * cnt;
            if (!ONE || r >= RP) {
                k_next = load(a.k_new, a.k_stride, t, h);
                v_next = load(a.v_new, a.v_stride, t, h);
            }
            const u32x4 k_raw = k_next, v_raw = v_next;
            const int64_t page_head = int64_t(id) * a.cache.n_kv_heads + h0 + h;
            put(key(k_raw, t), false, page_of(a.cache.k_pool, h), page_head, slot_lo + t);
            put(S::encode(v_raw), true, page_of(a.cache.v_pool, h), page_head, slot_lo + t);
        }
        return;
    }
    // a whole page: HEADS heads per pass, values through an image of their pages in LDS (two images in turn: one barrier per pass)
    const int t = row % kPage, sub = row / kPage;
    if (sub < n_heads) {
        k_next = load(a.k_new, a.k_stride, t, sub);
        v_next = load(a.v_new, a.v_stride, t, sub);
    }
    for (int h = 0, turn = 0; h < n_heads; h += HEADS, turn ^= 1) {
        uint8_t* img = image + turn * (HEADS * PADDED);
        const int mine = h + sub;
        if (mine < n_heads) {
            const u32x4 k_raw = k_next, v_raw = v_next;
            if (mine + HEADS < n_heads) {
                k_next = load(a.k_new, a.k_stride, t, mine + HEADS);
                v_next = load(a.v_new, a.v_stride, t, mine + HEADS);
            }
            const int64_t page_head = int64_t(id) * a.cache.n_kv_heads + h0 + mine;
            put(S::encode(v_raw), true, img + sub * PADDED + GAP * c, page_head, t);
            put(key(k_raw, t), false, page_of(a.cache.k_pool, mine), page_head, t);
        }
        __syncthreads();
        // (heads of a page lie one behind the other: the image is one run of bytes)
        constexpr int SHARE = HEADS * IMAGE / kRowsThreads;
        const int at = int(threadIdx.x) * SHARE;
        if (h + at / IMAGE < n_heads) {
            uint8_t* dst = page_of(a.cache.v_pool, h) + at;
            const uint8_t* src = img + at + GAP * (at / RUN);
            if constexpr (SHARE == 16) *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(src);
            else if constexpr (SHARE == 8) *reinterpret_cast<u32x2*>(dst) = *reinterpret_cast<const u32x2*>(src);
            else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(src);
        }
    }
}

__global__ void append_rows_len_kernel(int32_t* __restrict__ appended_len, const int32_t* __restrict__ n_new, int max_new, int batch, int capacity) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= batch) return;
    const int start = min(max(appended_len[b], 0), capacity);
    const int n = n_new ? min(max(n_new[b], 0), max_new) : max_new;
    appended_len[b] = start + min(n, capacity - start);
}

// pages of a sequence that n consecutive tokens may touch: the first of them in a page's last slot at worst, and no more than there are
inline int pages_touched(int n, const st_kv_cache& c) {
    return int(std::min<int64_t>((int64_t(n) - 2 + kPage) / kPage + 1, c.max_pages_per_seq));
}

// Workgroups to aim at by splitting the heads of a page: 64 sentences of up to 190 tokens (900 pages) 17 us, with 512 24, with 4,096 19 (the page's
// angles are evaluated by each).
constexpr int kAppendWorkgroups = 2048;

st_status append_rows(const char* who, const st_kv_cache& c, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                      const int32_t* start_len, const int32_t* n_new, int max_new, int batch, const void* k_weight, double eps,
                      const RopeTable* rope, hipStream_t s) {
    PagesArgs a{};
    a.cache = cache_view(c);
    a.k_new = static_cast<const uint16_t*>(k_new);
    a.v_new = static_cast<const uint16_t*>(v_new);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.start_len = start_len;
    a.n_new = n_new;
    a.max_new = max_new;
    a.touched = pages_touched(max_new, c);
    a.k_weight = static_cast<const uint16_t*>(k_weight);
    a.eps = eps;
    a.rotate = rope != nullptr;
    if (rope) a.rope = *rope;
    if (rope && max_new > 1) {
        // (128 calls of cos and sin: kept as the table itself is)
        static thread_local double kept_f[64];
        static thread_local double2 kept[64];
        if (memcmp(kept_f, rope->f, sizeof(kept_f)) != 0) {
            for (int i = 0; i < 64; ++i) kept[i] = double2{cos(rope->f[i]), sin(rope->f[i])};
            memcpy(kept_f, rope->f, sizeof(kept_f));
        }
        memcpy(a.step, kept, sizeof(kept));
    }
    // all heads of a page in one workgroup, split where that leaves the chip's compute units without work
    const int hkv = c.n_kv_heads;
    const int64_t pages = int64_t(batch) * a.touched;
    a.head_groups = int(std::min<int64_t>(hkv, std::max<int64_t>(1, kAppendWorkgroups / pages)));
    const bool one_reader = a.touched == 1 && max_new == 1;
    if (one_reader) a.head_groups = 1;
    a.heads = (hkv + a.head_groups - 1) / a.head_groups;
    a.head_groups = (hkv + a.heads - 1) / a.heads;
    // the new lengths go in with this launch where nobody else reads the old ones
    a.write_len = start_len || one_reader;
    const int64_t blocks = pages * a.head_groups;
    if (blocks > 0x7fffffff) return fail(ST_ERR_SHAPE, "%s: grid too large", who);
    // (LDS images: 16 tokens x D dims x HEADS heads and the gaps, the same bytes for 64 dims and two heads as for 128 and one)
    auto go = [&](auto format, int image) {
        constexpr int FMT = decltype(format)::value;
        const size_t smem = (rope ? size_t(kPage) * (a.rope.rot / 2) * sizeof(double2) : 0) + size_t(2 * image)
                          + (rope && FMT != ST_BF16 ? (size_t(kPage) * (a.rope.rot / 2) * 3 + 16) * sizeof(float) : 0);
        auto launch = [&](auto kernel, const auto& args) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRowsThreads), smem, s, args); };
        const RowsArgs& one = a;
        if (max_new == 1) {
            if (c.head_dim == 64) launch(append_rows_kernel<FMT, 64, RowsArgs>, one); else launch(append_rows_kernel<FMT, 128, RowsArgs>, one);
        } else {
            if (c.head_dim == 64) launch(append_rows_kernel<FMT, 64, PagesArgs>, a); else launch(append_rows_kernel<FMT, 128, PagesArgs>, a);
        }
    };
    const int values = 16 * 128;
    if (c.dtype == ST_MXFP4) go(std::integral_constant<int, ST_MXFP4>{}, values / 2);
    else if (c.dtype == ST_FP8_E4M3) go(std::integral_constant<int, ST_FP8_E4M3>{}, values + 256);
    else go(std::integral_constant<int, ST_BF16>{}, 2 * values + 256);
    ST_LAUNCH_CHECK("append_rows_kernel");
    if (!a.write_len) {
        hipLaunchKernelGGL(append_rows_len_kernel, dim3((unsigned(batch) + 255u) / 256u), dim3(256), 0, s, c.appended_len, n_new, max_new, batch, c.max_pages_per_seq * kPage);
        ST_LAUNCH_CHECK("append_rows_len_kernel");
    }
    return ST_OK;
}

// ---- rows read back --------------------------------------------------------------------------------------------------
struct ReadArgs {
    CacheView cache;
    uint16_t* k_out;             // [batch][max_n][n_kv_heads][D]
    uint16_t* v_out;
    const int32_t* first;        // [batch], or null: 0
    const int32_t* n;            // [batch], or null: max_n
    int max_n, touched;
    int heads, head_groups;
};

// the two codes of byte `byte` as bf16 times the power of two of an E8M0 byte (255: NaN)
__device__ __forceinline__ uint32_t pair_of_codes(uint32_t w, uint32_t scale, int byte) { return fp4_pair(w, __uint_as_float(scale << 23), byte); }

// What a thread reads of a page of one head, ahead of its use: a share of the values (eight, at (slot, dim) of its own) and the eight dims 8 c .. of
// the key of its slot, with their scales.
template <int FMT, int D>
struct Stored;

template <int D>
struct Stored<ST_MXFP4, D> {
    static constexpr int G = D / 32;
    uint32_t v, vs, k, ks;
    __device__ __forceinline__ void load(const CacheView& cv, int64_t page_head, int share, int slot, int c) {
        const uint8_t* kp = reinterpret_cast<const uint8_t*>(cv.k_pool) + page_head * (D * 8);
        const uint8_t* vp = reinterpret_cast<const uint8_t*>(cv.v_pool) + page_head * (D * 8);
        const uint8_t* sp = reinterpret_cast<const uint8_t*>(cv.k_scale) + page_head * D;
        v = *reinterpret_cast<const uint32_t*>(vp + 4 * share);
        vs = *reinterpret_cast<const uint32_t*>(sp + D / 2 + ((share / (16 * G)) * G + share % G) * 4);
        k = *reinterpret_cast<const uint32_t*>(kp + ((c >> 2) * kPage + slot) * 16 + 4 * (c & 3));
        ks = sp[(c >> 2) * kPage + slot];
    }
    // dword `share`: slots 4 q .. + 3 of dims 32 g + m and 32 g + 16 + m
    template <typename Each>
    __device__ __forceinline__ void values(int share, Each each) const {
        const int g = share % G, m = (share / G) % 16, q = share / (16 * G);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t w = pair_of_codes(v, (vs >> (8 * t)) & 255u, t);
            each(4 * q + t, 32 * g + m, uint16_t(w));
            each(4 * q + t, 32 * g + 16 + m, uint16_t(w >> 16));
        }
    }
    __device__ __forceinline__ u32x4 key() const { return u32x4{pair_of_codes(k, ks, 0), pair_of_codes(k, ks, 1), pair_of_codes(k, ks, 2), pair_of_codes(k, ks, 3)}; }
};

template <int D>
struct Stored<ST_FP8_E4M3, D> {
    u32x2 v, k;
    f32x4 vs[2];
    float ks;
    __device__ __forceinline__ void load(const CacheView& cv, int64_t page_head, int share, int slot, int c) {
        v = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(cv.v_pool) + page_head * (D * kPage) + 8 * share);
        const f32x4* sc = reinterpret_cast<const f32x4*>(cv.v_scale + page_head * kPage + 8 * (share & 1));
        vs[0] = sc[0];
        vs[1] = sc[1];
        k = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(cv.k_pool) + page_head * (D * kPage) + ((c >> 1) * kPage + slot) * 16 + 8 * (c & 1));
        ks = cv.k_scale[page_head * kPage + slot];
    }
    static __device__ __forceinline__ void unpack(const u32x2& w, float (&f)[8]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f[4 * u] = __builtin_amdgcn_cvt_f32_fp8(w[u], 0);
            f[4 * u + 1] = __builtin_amdgcn_cvt_f32_fp8(w[u], 1);
            f[4 * u + 2] = __builtin_amdgcn_cvt_f32_fp8(w[u], 2);
            f[4 * u + 3] = __builtin_amdgcn_cvt_f32_fp8(w[u], 3);
        }
    }
    // eight slots of dim share / 2
    template <typename Each>
    __device__ __forceinline__ void values(int share, Each each) const {
        float f[8];
        unpack(v, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) each(8 * (share & 1) + e, share / 2, f32_to_bf16_bits(f[e] * vs[e / 4][e & 3]));
    }
    __device__ __forceinline__ u32x4 key() const {
        float f[8];
        unpack(k, f);
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pair_bf16(f[2 * i] * ks, f[2 * i + 1] * ks);
        return r;
    }
};

template <int D>
struct Stored<ST_BF16, D> {
    u32x4 v, k;
    __device__ __forceinline__ void load(const CacheView& cv, int64_t page_head, int share, int slot, int c) {
        v = *reinterpret_cast<const u32x4*>(cv.v_pool + page_head * (D * kPage) + 8 * share);
        k = *reinterpret_cast<const u32x4*>(cv.k_pool + page_head * (D * kPage) + (c * kPage + slot) * 8);
    }
    template <typename Each>
    __device__ __forceinline__ void values(int share, Each each) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) each(8 * (share & 1) + e, share / 2, uint16_t(v[e / 2] >> (16 * (e & 1))));
    }
    __device__ __forceinline__ u32x4 key() const { return k; }
};

template <int FMT, int D>
__global__ __launch_bounds__(kRowsThreads) void read_rows_kernel(ReadArgs a) {
    constexpr int L = D / 8, RP = kRowsThreads / L, HEADS = RP / kPage;
    constexpr int ROW = D + 8;                                   // (padded: slots start in different banks)
    __shared__ __align__(16) uint16_t s_v[2][HEADS][kPage][ROW];
    const int group = int(blockIdx.x) % a.head_groups, pi = (int(blockIdx.x) / a.head_groups) % a.touched, b = int(blockIdx.x) / (a.head_groups * a.touched);
    const int capacity = a.cache.max_pages * kPage;
    const int first = min(max(a.first ? a.first[b] : 0, 0), capacity);
    const int n = min(a.n ? min(max(a.n[b], 0), a.max_n) : a.max_n, capacity - first);
    const int page = first / kPage + pi;
    const int lo = max(first, page * kPage), hi = min(first + n, (page + 1) * kPage);
    if (lo >= hi) return;
    const int id = a.cache.page_table[int64_t(b) * a.cache.max_pages + page];
    if (id < 0 || id >= a.cache.n_pages) return;
    const int h0 = group * a.heads, n_heads = min(a.heads, a.cache.n_kv_heads - h0);
    const int c = int(threadIdx.x) % L, slot = (int(threadIdx.x) / L) % kPage, sub = int(threadIdx.x) / (L * kPage);
    const int share = int(threadIdx.x) % (L * kPage);            // of a head's page: D * 16 values / 8
    const int tok = page * kPage + slot;
    const bool wanted = tok >= lo && tok < hi;
    // (the next heads' bytes are under way while these are sorted)
    const int64_t first_head = int64_t(id) * a.cache.n_kv_heads + h0;
    Stored<FMT, D> next;
    if (sub < n_heads) next.load(a.cache, first_head + sub, share, slot, c);
    for (int h = 0, turn = 0; h < n_heads; h += HEADS, turn ^= 1) {
        const int mine = h + sub;
        const int64_t at = ((int64_t(b) * a.max_n + (tok - first)) * a.cache.n_kv_heads + h0 + mine) * D + 8 * c;
        if (mine < n_heads) {
            const Stored<FMT, D> now = next;
            if (mine + HEADS < n_heads) next.load(a.cache, first_head + mine + HEADS, share, slot, c);
            now.values(share, [&](int s, int d, uint16_t v) { s_v[turn][sub][s][d] = v; });
            if (wanted) *reinterpret_cast<u32x4*>(a.k_out + at) = now.key();
        }
        __syncthreads();
        if (mine < n_heads && wanted) *reinterpret_cast<u32x4*>(a.v_out + at) = *reinterpret_cast<const u32x4*>(&s_v[turn][sub][slot][8 * c]);
    }
}

// (There are no angles to share: the same sentences are read in 9.9 us, with 8,192 in 11.5.)
constexpr int kReadWorkgroups = 4096;

// what both directions ask of a cache and of the rows beside it
static st_status check_rows_call(const char* who, const st_dual_cache* caches, st_stream_kind which, const void* k, const void* v, int32_t max_rows,
                                 int32_t batch) {
    if (!caches || (max_rows > 0 && (!k || !v))) return fail(ST_ERR_INVALID_ARG, "%s: null pointer", who);
    if (which != ST_SOURCE && which != ST_REASONING) return fail(ST_ERR_INVALID_ARG, "%s: which = %d", who, int(which));
    const st_status r = check_cache(which == ST_SOURCE ? caches->source : caches->reasoning, who, which == ST_SOURCE ? "source" : "reasoning", true, true);
    if (r != ST_OK) return r;
    if (!aligned16(k) || !aligned16(v)) return fail(ST_ERR_INVALID_ARG, "%s: key and value rows must be 16-byte aligned", who);
    if (batch <= 0 || max_rows < 0) return fail(ST_ERR_INVALID_ARG, "%s: bad sizes", who);
    return ST_OK;
}

}  // namespace st

using namespace st;

extern "C" st_status st_kv_append_norm_rope(const st_dual_cache* caches, st_stream_kind which, const void* k_new, int64_t k_stride, const void* v_new,
                                            int64_t v_stride, const int32_t* start_len, const int32_t* n_new, int32_t max_new, int32_t batch,
                                            int32_t host_len_upper_bound, const void* k_weight, double eps, const st_rope_spec* spec,
                                            void* hip_stream) {
    const char* who = "st_kv_append_norm_rope";
    st_status r = check_rows_call(who, caches, which, k_new, v_new, max_new, batch);
    if (r != ST_OK) return r;
    const st_kv_cache& c = which == ST_SOURCE ? caches->source : caches->reasoning;
    if (!c.appended_len) return fail(ST_ERR_INVALID_ARG, "%s: appended_len is null", who);
    if (start_len == c.appended_len) start_len = nullptr;       // (the same lengths, which the call is about to change)
    if (start_len && n_new == c.appended_len) return fail(ST_ERR_INVALID_ARG, "%s: n_new is the cache's appended_len, which the call writes", who);
    const int64_t dense = int64_t(c.n_kv_heads) * c.head_dim;
    if (k_stride < dense || v_stride < dense) return fail(ST_ERR_SHAPE, "%s: a token stride of %lld elements for %d heads of %d", who, (long long)std::min(k_stride, v_stride), c.n_kv_heads, c.head_dim);
    if (k_stride % 8 != 0 || v_stride % 8 != 0) return fail(ST_ERR_INVALID_ARG, "%s: token strides must be multiples of 16 bytes", who);
    const int64_t capacity = int64_t(c.max_pages_per_seq) * kPage;
    if (host_len_upper_bound < 0 || host_len_upper_bound > capacity)
        return fail(ST_ERR_CAPACITY, "%s: length bound %d exceeds the page table (%lld tokens per sequence)", who, host_len_upper_bound, (long long)capacity);
    if (!aligned16(k_weight)) return fail(ST_ERR_INVALID_ARG, "%s: k_weight must be 16-byte aligned", who);
    if (!(eps >= 0.0 && eps < HUGE_VAL)) return fail(ST_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
    RopeTable rope;
    if (spec) {
        r = make_rope_table(who, spec, c.head_dim, &rope);
        if (r != ST_OK) return r;
    }
    if (max_new == 0 && !start_len) return ST_OK;
    return append_rows(who, c, k_new, k_stride, v_new, v_stride, start_len, n_new, max_new, batch, k_weight, eps, spec ? &rope : nullptr,
                       static_cast<hipStream_t>(hip_stream));
}

extern "C" st_status st_kv_read(const st_dual_cache* caches, st_stream_kind which, void* k_out, void* v_out, const int32_t* first, const int32_t* n,
                                int32_t max_n, int32_t batch, void* hip_stream) {
    const char* who = "st_kv_read";
    const st_status r = check_rows_call(who, caches, which, k_out, v_out, max_n, batch);
    if (r != ST_OK) return r;
    if (max_n == 0) return ST_OK;
    const st_kv_cache& c = which == ST_SOURCE ? caches->source : caches->reasoning;
    ReadArgs a{};
    a.cache = cache_view(c);
    a.k_out = static_cast<uint16_t*>(k_out);
    a.v_out = static_cast<uint16_t*>(v_out);
    a.first = first;
    a.n = n;
    a.max_n = max_n;
    a.touched = pages_touched(max_n, c);
    const int64_t pages = int64_t(batch) * a.touched;
    const int hkv = c.n_kv_heads;
    a.head_groups = int(std::min<int64_t>(hkv, std::max<int64_t>(1, kReadWorkgroups / pages)));
    a.heads = (hkv + a.head_groups - 1) / a.head_groups;
    a.head_groups = (hkv + a.heads - 1) / a.heads;
    const int64_t blocks = pages * a.head_groups;
    if (blocks > 0x7fffffff) return fail(ST_ERR_SHAPE, "%s: grid too large", who);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRowsThreads), 0, static_cast<hipStream_t>(hip_stream), a); };
    if (c.dtype == ST_MXFP4) {
        if (c.head_dim == 64) go(read_rows_kernel<ST_MXFP4, 64>); else go(read_rows_kernel<ST_MXFP4, 128>);
    } else if (c.dtype == ST_FP8_E4M3) {
        if (c.head_dim == 64) go(read_rows_kernel<ST_FP8_E4M3, 64>); else go(read_rows_kernel<ST_FP8_E4M3, 128>);
    } else {
        if (c.head_dim == 64) go(read_rows_kernel<ST_BF16, 64>); else go(read_rows_kernel<ST_BF16, 128>);
    }
    ST_LAUNCH_CHECK("read_rows_kernel");
    return ST_OK;
}
