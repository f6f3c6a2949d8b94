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
// and the same row would not always be stored alike.  fp64 runs at the rate of unpacked fp32 here, so it costs registers, not time.
#include <math.h>

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

// 64 bits rounded to bf16 in ONE rounding: to 32 bits with the last bit set if anything was lost, then to nearest even
__device__ __forceinline__ uint16_t f64_to_bf16_bits(double x) {
    const float f = float(x);
    uint32_t u = __float_as_uint(f);
    if (double(f) != x) {
        if (fabs(double(f)) > fabs(x)) u -= 1;
        u |= 1u;
    }
    return f32_to_bf16_bits(__uint_as_float(u));
}

constexpr int kScaleExpLeast = -100;             // of 8-bit rows and 4-bit blocks alike

// Largest magnitude (as bf16 bits, non-finite above all) of a lane's eight values, over LANES neighbouring lanes
template <int LANES>
__device__ __forceinline__ uint32_t row_top(const u32x4& x) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
    auto fold = [&](auto ctrl) { top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), decltype(ctrl)::value, 0xf, 0xf, true))); };
    fold(std::integral_constant<int, 0xb1>{});
    fold(std::integral_constant<int, 0x4e>{});
    if constexpr (LANES >= 8) fold(std::integral_constant<int, 0x141>{});
    if constexpr (LANES >= 16) fold(std::integral_constant<int, 0x140>{});
    return top;
}
// The smallest k from -100 on with (bf16 bits) top <= m 2^(e + k), m = 1 + m128 / 128; 0 for top = 0
__device__ __forceinline__ int scale_exponent(uint32_t top, int m128, int e) {
    if (top == 0) return 0;
    return max(int(top >> 7) - 127 - e + (int(top & 127u) > m128 ? 1 : 0), kScaleExpLeast);
}

// Storage formats.  A lane stores its eight key dims (8 c ..) of slot s, a thread of a whole page's image its share of V.
//   PIECE bytes a lane holds of a row; v_at(slot, d) byte of value element in a page of one head
template <int FMT, int D>
struct Store;

template <int D>
struct Store<ST_BF16, D> {
    static constexpr int PIECE = 16;
    static __device__ __forceinline__ u32x4 code(const u32x4& x, bool, const CacheView&, int64_t, int, int) { return x; }
    static __device__ __forceinline__ void put_key(uint8_t* page, int slot, int c, const u32x4& p) { *reinterpret_cast<u32x4*>(page + (c * kPage + slot) * 16) = p; }
    static __device__ __forceinline__ void put_value(uint8_t* page, int slot, int c, const u32x4& p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) *reinterpret_cast<uint16_t*>(page + ((8 * c + e) * kPage + slot) * 2) = uint16_t(p[e / 2] >> (16 * (e & 1)));
    }
};

template <int D>
struct Store<ST_FP8_E4M3, D> {
    static constexpr int PIECE = 8;
    // codes of a lane's eight dims, the row's scale written by the row's first lane
    static __device__ __forceinline__ u32x4 code(const u32x4& x, bool value, const CacheView& cv, int64_t page_head, int slot, int c) {
        const uint32_t top = row_top<D / 8>(x);
        // (448 = 1.75 * 2^8.  A row with an infinite or undefined element: that element's code is NaN, the scale the largest there is)
        const int k = scale_exponent(min(top, 0x7f7fu), 96, 8);
        if (c == 0) (value ? cv.v_scale : cv.k_scale)[page_head * kPage + slot] = ldexpf(1.f, k);
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = ldexpf(__uint_as_float(x[i] << 16), -k), hi = ldexpf(__uint_as_float(x[i] & 0xffff0000u), -k);
            if (i & 1) w[i / 2] = __builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, w[i / 2], true);
            else w[i / 2] = __builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, w[i / 2], false);
        }
        return u32x4{w[0], w[1], 0u, 0u};
    }
    static __device__ __forceinline__ void put_key(uint8_t* page, int slot, int c, const u32x4& p) {
        *reinterpret_cast<u32x2*>(page + ((c >> 1) * kPage + slot) * 16 + 8 * (c & 1)) = u32x2{p[0], p[1]};
    }
    static __device__ __forceinline__ void put_value(uint8_t* page, int slot, int c, const u32x4& p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) page[(8 * c + e) * kPage + slot] = uint8_t(p[e / 4] >> (8 * (e & 3)));
    }
};

// 4 bits: see st_kv_cache.  A value byte holds dims d and d + 16 of one token, so that no byte is shared between tokens: the lanes of dims
// 8 c and 8 (c ^ 2) exchange codes, and each writes four of the eight bytes that the two have in common.
template <int D>
struct Store<ST_MXFP4, D> {
    static constexpr int PIECE = 4;
    static __device__ __forceinline__ u32x4 code(const u32x4& x, bool value, const CacheView& cv, int64_t page_head, int slot, int c) {
        const uint32_t top = row_top<4>(x);                  // a block of 32 dims: four lanes
        const bool bad = top >= 0x7f80u;
        const int k = bad ? 0 : scale_exponent(top, 64, 2);  // 6 = 1.5 * 2^2
        if ((c & 3) == 0) {
            uint8_t* scales = reinterpret_cast<uint8_t*>(cv.k_scale) + page_head * D;
            const int at = value ? D / 2 + ((slot >> 2) * (D / 32) + (c >> 2)) * 4 + (slot & 3) : (c >> 2) * kPage + slot;
            scales[at] = bad ? uint8_t(255) : uint8_t(k + 127);
        }
        const float scale = __uint_as_float(uint32_t(k + 127) << 23);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[1] << 16), __uint_as_float(x[1] & 0xffff0000u), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[2] << 16), __uint_as_float(x[2] & 0xffff0000u), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[3] << 16), __uint_as_float(x[3] & 0xffff0000u), scale, 3);
        return u32x4{bad ? 0u : w, 0u, 0u, 0u};
    }
    static __device__ __forceinline__ void put_key(uint8_t* page, int slot, int c, const u32x4& p) {
        *reinterpret_cast<uint32_t*>(page + ((c >> 2) * kPage + slot) * 16 + 4 * (c & 3)) = p[0];
    }
    static __device__ __forceinline__ void put_value(uint8_t* page, int slot, int c, const u32x4& p) {
        const uint32_t mine = p[0], other = uint32_t(__builtin_amdgcn_update_dpp(0, int(mine), 0x4e, 0xf, 0xf, true));      // lane c ^ 2
        const bool high = (c & 2) != 0;                     // this lane holds the dims 16 further on
        const uint32_t lo = high ? other : mine, hi = high ? mine : other;
        const int first = high ? 4 : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = first + i, m = 8 * (c & 1) + e;   // dim within sixteen
            page[((slot >> 2) * 16 + m) * (D / 8) + (c >> 2) * 4 + (slot & 3)] = uint8_t(((lo >> (4 * e)) & 15u) | (((hi >> (4 * e)) & 15u) << 4));
        }
    }
};

// A key row's eight dims in a lane, normalised and rotated in 64 bits
template <int D>
__device__ __forceinline__ u32x4 transform_key(const u32x4& raw, const RowsArgs& a, const u32x4& w_raw, const double2* table) {
    constexpr int L = D / 8;
    const int c = int(threadIdx.x) % L, half = a.rope.rot / 2;
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
        const double r = 1.0 / sqrt(row_sum<L>(ss) * (1.0 / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] *= r * double(__uint_as_float(w_raw[i] << 16));
            x[2 * i + 1] *= r * double(__uint_as_float(w_raw[i] & 0xffff0000u));
        }
    }
    if (a.rotate) {
        const bool turned = 8 * c < a.rope.rot;
        if (a.rope.interleaved) {
            if (turned) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double2 r = table[4 * c + i];
                    const double lo = x[2 * i], hi = x[2 * i + 1];
                    x[2 * i] = lo * r.x - hi * r.y;
                    x[2 * i + 1] = hi * r.x + lo * r.y;
                }
            }
        } else {
            const bool high = 8 * c >= half;
            const int partner = (int(threadIdx.x) & 63) + (turned ? (high ? -half / 8 : half / 8) : 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double other = __shfl(x[i], partner);
                if (turned) {
                    const double2 r = table[(high ? 8 * c - half : 8 * c) + i];
                    x[i] = x[i] * r.x + other * (high ? r.y : -r.y);
                }
            }
        }
    }
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = uint32_t(f64_to_bf16_bits(x[2 * i])) | (uint32_t(f64_to_bf16_bits(x[2 * i + 1])) << 16);
    return out;
}

constexpr int kRowsThreads = 256;

template <int FMT, int D>
__global__ __launch_bounds__(kRowsThreads) void append_rows_kernel(RowsArgs a) {
    using S = Store<FMT, D>;
    constexpr int L = D / 8, RP = kRowsThreads / L, HEADS = RP / kPage;      // rows, whole pages of a head per pass
    constexpr int IMAGE = D * kPage * S::PIECE / 8;                          // bytes of a page of one head
    extern __shared__ __align__(16) unsigned char smem[];
    double2* table = reinterpret_cast<double2*>(smem);                       // [16][rot / 2] (cos, sin) times a
    uint8_t* image = smem + (a.rotate ? kPage * (a.rope.rot / 2) * sizeof(double2) : 0);         // [2][HEADS][IMAGE]
    const int group = int(blockIdx.x) % a.head_groups, pi = (int(blockIdx.x) / a.head_groups) % a.touched, b = int(blockIdx.x) / (a.head_groups * a.touched);
    const int capacity = a.cache.max_pages * kPage;
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
    const int id = a.cache.page_table[int64_t(b) * a.cache.max_pages + page];
    if (id < 0 || id >= a.cache.n_pages) return;                             // never write outside the pool
    const int slot_lo = lo - page * kPage, cnt = hi - lo;
    const int h0 = group * a.heads, n_heads = min(a.heads, a.cache.n_kv_heads - h0);
    const int c = int(threadIdx.x) % L, row = int(threadIdx.x) / L;
    const int64_t tok0 = int64_t(b) * a.max_new + (lo - start);

    u32x4 w_raw = {0u, 0u, 0u, 0u};
    if (a.k_weight) w_raw = *reinterpret_cast<const u32x4*>(a.k_weight + 8 * c);
    const int half = a.rope.rot / 2;
    if (a.rotate) {
        for (int w = int(threadIdx.x); w < cnt * half; w += kRowsThreads) {
            const int t = w / half, i = w - t * half;
            const double rev = double(lo + t) * a.rope.f[i] * 0.15915494309189535;       // angle / 2 pi; a token's index is its position id
            double sn, cs;
            sincospi(2.0 * (rev - rint(rev)), &sn, &cs);
            table[w] = double2{cs * a.rope.a, sn * a.rope.a};
        }
        __syncthreads();
    }
    auto load = [&](const uint16_t* src, int64_t stride, int t, int h) { return *reinterpret_cast<const u32x4*>(src + (tok0 + t) * stride + (h0 + h) * D + 8 * c); };
    auto page_of = [&](uint16_t* pool, int h) { return reinterpret_cast<uint8_t*>(pool) + (int64_t(id) * a.cache.n_kv_heads + h0 + h) * IMAGE; };
    auto key = [&](const u32x4& raw, int t) { return a.k_weight || a.rotate ? transform_key<D>(raw, a, w_raw, table + t * half) : raw; };

    if (cnt < kPage) {
        // part of a page: rows (head, token) in turn, straight to their places
        for (int r = row; r < cnt * n_heads; r += RP) {
            const int h = r / cnt, t = r - h * cnt;
            const u32x4 k_raw = load(a.k_new, a.k_stride, t, h), v_raw = load(a.v_new, a.v_stride, t, h);
            const int64_t page_head = int64_t(id) * a.cache.n_kv_heads + h0 + h;
            S::put_key(page_of(a.cache.k_pool, h), slot_lo + t, c, S::code(key(k_raw, t), false, a.cache, page_head, slot_lo + t, c));
            S::put_value(page_of(a.cache.v_pool, h), slot_lo + t, c, S::code(v_raw, true, a.cache, page_head, slot_lo + t, c));
        }
        return;
    }
    // a whole page: HEADS heads per pass, values through an image of their pages in LDS (two images in turn: one barrier per pass)
    const int t = row % kPage, sub = row / kPage;
    for (int h = 0, turn = 0; h < n_heads; h += HEADS, turn ^= 1) {
        uint8_t* img = image + turn * (HEADS * IMAGE);
        const int mine = h + sub;
        if (mine < n_heads) {
            const u32x4 k_raw = load(a.k_new, a.k_stride, t, mine), v_raw = load(a.v_new, a.v_stride, t, mine);
            const int64_t page_head = int64_t(id) * a.cache.n_kv_heads + h0 + mine;
            S::put_value(img + sub * IMAGE, t, c, S::code(v_raw, true, a.cache, page_head, t, c));
            S::put_key(page_of(a.cache.k_pool, mine), t, c, S::code(key(k_raw, t), false, a.cache, page_head, t, c));
        }
        __syncthreads();
        // (heads of a page lie one behind the other: the image is one run of bytes)
        constexpr int SHARE = HEADS * IMAGE / kRowsThreads;
        const int at = int(threadIdx.x) * SHARE;
        if (h + at / IMAGE < n_heads) {
            uint8_t* dst = page_of(a.cache.v_pool, h) + at;
            if constexpr (SHARE == 16) *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(img + at);
            else if constexpr (SHARE == 8) *reinterpret_cast<u32x2*>(dst) = *reinterpret_cast<const u32x2*>(img + at);
            else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(img + at);
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

st_status append_rows(const char* who, const st_kv_cache& c, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                      const int32_t* start_len, const int32_t* n_new, int max_new, int batch, const void* k_weight, double eps,
                      const RopeTable* rope, hipStream_t s) {
    RowsArgs a{};
    a.cache = cache_view(c);
    a.k_new = static_cast<const uint16_t*>(k_new);
    a.v_new = static_cast<const uint16_t*>(v_new);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.start_len = start_len;
    a.n_new = n_new;
    a.max_new = max_new;
    a.touched = (max_new - 2 + kPage) / kPage + 1;               // (the first token in a page's last slot at worst)
    a.k_weight = static_cast<const uint16_t*>(k_weight);
    a.eps = eps;
    a.rotate = rope != nullptr;
    if (rope) a.rope = *rope;
    // all heads of a page in one workgroup, split where that leaves the chip's compute units without work
    const int hkv = c.n_kv_heads;
    const int64_t pages = int64_t(batch) * a.touched;
    a.head_groups = int(std::min<int64_t>(hkv, std::max<int64_t>(1, 512 / std::max<int64_t>(pages, 1))));
    const bool one_reader = a.touched == 1 && max_new == 1;
    if (one_reader) a.head_groups = 1;
    a.heads = (hkv + a.head_groups - 1) / a.head_groups;
    a.head_groups = (hkv + a.heads - 1) / a.heads;
    // the new lengths go in with this launch where nobody else reads the old ones
    a.write_len = start_len || one_reader;
    const int64_t blocks = pages * a.head_groups;
    if (blocks > 0x7fffffff) return fail(ST_ERR_SHAPE, "%s: grid too large", who);
    auto go = [&](auto kernel, int image) {
        const size_t smem = (rope ? size_t(kPage) * (a.rope.rot / 2) * sizeof(double2) : 0) + size_t(2 * image);
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRowsThreads), smem, s, a);
    };
    // (LDS images: 16 tokens x D dims x HEADS heads, the same bytes for 64 dims and two heads as for 128 and one)
    const int values = 16 * 128;
    if (c.dtype == ST_MXFP4) {
        if (c.head_dim == 64) go(append_rows_kernel<ST_MXFP4, 64>, values / 2); else go(append_rows_kernel<ST_MXFP4, 128>, values / 2);
    } else if (c.dtype == ST_FP8_E4M3) {
        if (c.head_dim == 64) go(append_rows_kernel<ST_FP8_E4M3, 64>, values); else go(append_rows_kernel<ST_FP8_E4M3, 128>, values);
    } else {
        if (c.head_dim == 64) go(append_rows_kernel<ST_BF16, 64>, 2 * values); else go(append_rows_kernel<ST_BF16, 128>, 2 * values);
    }
    ST_LAUNCH_CHECK("append_rows_kernel");
    if (!a.write_len) {
        hipLaunchKernelGGL(append_rows_len_kernel, dim3((batch + 255) / 256), dim3(256), 0, s, c.appended_len, n_new, max_new, batch, c.max_pages_per_seq * kPage);
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

// E8M0 as fp32 (255: NaN)
__device__ __forceinline__ float e8m0(uint32_t b) { return __uint_as_float(b == 255u ? 0x7fc00000u : b << 23); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    bf16x2 r;
    r[0] = (__bf16)lo;
    r[1] = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ float e2m1(uint32_t code) {
    const uint32_t m = code & 7u;
    const float v = m < 2 ? 0.5f * float(m) : ldexpf(float(2 + (m & 1u)), int(m >> 1) - 2);
    return code & 8u ? -v : v;
}

// A thread's share of a page of values of one head: eight values, at (slot, dim) of its own, as fp32 times the scale
template <int FMT, int D, typename Each>
__device__ __forceinline__ void read_values(const CacheView& cv, const uint8_t* page, int64_t page_head, int share, Each each) {
    if constexpr (FMT == ST_MXFP4) {
        // dword `share`: slots 4 q .. + 3 of dims 32 g + m and 32 g + 16 + m
        constexpr int G = D / 32;
        const int g = share % G, m = (share / G) % 16, q = share / (16 * G);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(page + 4 * share);
        const uint32_t sc = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(cv.k_scale) + page_head * D + D / 2 + (q * G + g) * 4);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float scale = e8m0((sc >> (8 * t)) & 255u);
            each(4 * q + t, 32 * g + m, e2m1((w >> (8 * t)) & 15u) * scale);
            each(4 * q + t, 32 * g + 16 + m, e2m1((w >> (8 * t + 4)) & 15u) * scale);
        }
    } else {
        // eight slots of dim share / 2
        const int d = share / 2, s0 = 8 * (share & 1);
        if constexpr (FMT == ST_FP8_E4M3) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(page + 8 * share);
            const float* sc = cv.v_scale + page_head * kPage + s0;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                each(s0 + 4 * u, d, __builtin_amdgcn_cvt_f32_fp8(w[u], 0) * sc[4 * u]);
                each(s0 + 4 * u + 1, d, __builtin_amdgcn_cvt_f32_fp8(w[u], 1) * sc[4 * u + 1]);
                each(s0 + 4 * u + 2, d, __builtin_amdgcn_cvt_f32_fp8(w[u], 2) * sc[4 * u + 2]);
                each(s0 + 4 * u + 3, d, __builtin_amdgcn_cvt_f32_fp8(w[u], 3) * sc[4 * u + 3]);
            }
        } else {
            const u32x4 w = *reinterpret_cast<const u32x4*>(page + 16 * share);
#pragma unroll
            for (int e = 0; e < 8; ++e) each(s0 + e, d, bf16_bits_to_f32(uint16_t(w[e / 2] >> (16 * (e & 1)))));
        }
    }
}

// eight dims (8 c ..) of a stored key
template <int FMT, int D>
__device__ __forceinline__ u32x4 read_key(const CacheView& cv, const uint8_t* page, int64_t page_head, int slot, int c) {
    if constexpr (FMT == ST_MXFP4) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(page + ((c >> 2) * kPage + slot) * 16 + 4 * (c & 3));
        const float scale = e8m0(reinterpret_cast<const uint8_t*>(cv.k_scale)[page_head * D + (c >> 2) * kPage + slot]);
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack_bf16(e2m1((w >> (8 * i)) & 15u) * scale, e2m1((w >> (8 * i + 4)) & 15u) * scale);
        return r;
    } else if constexpr (FMT == ST_FP8_E4M3) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(page + ((c >> 1) * kPage + slot) * 16 + 8 * (c & 1));
        const float scale = cv.k_scale[page_head * kPage + slot];
        u32x4 r;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            r[2 * u] = pack_bf16(__builtin_amdgcn_cvt_f32_fp8(w[u], 0) * scale, __builtin_amdgcn_cvt_f32_fp8(w[u], 1) * scale);
            r[2 * u + 1] = pack_bf16(__builtin_amdgcn_cvt_f32_fp8(w[u], 2) * scale, __builtin_amdgcn_cvt_f32_fp8(w[u], 3) * scale);
        }
        return r;
    } else {
        return *reinterpret_cast<const u32x4*>(page + (c * kPage + slot) * 16);
    }
}

template <int FMT, int D>
__global__ __launch_bounds__(kRowsThreads) void read_rows_kernel(ReadArgs a) {
    constexpr int L = D / 8, RP = kRowsThreads / L, HEADS = RP / kPage, IMAGE = D * kPage * Store<FMT, D>::PIECE / 8;
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
    for (int h = 0, turn = 0; h < n_heads; h += HEADS, turn ^= 1) {
        const int mine = h + sub;
        const int64_t page_head = int64_t(id) * a.cache.n_kv_heads + h0 + mine;
        const int64_t at = ((int64_t(b) * a.max_n + (tok - first)) * a.cache.n_kv_heads + h0 + mine) * D + 8 * c;
        if (mine < n_heads) {
            read_values<FMT, D>(a.cache, reinterpret_cast<const uint8_t*>(a.cache.v_pool) + page_head * IMAGE, page_head, share,
                                [&](int s, int d, float v) { s_v[turn][sub][s][d] = f32_to_bf16_bits(v); });
            if (wanted)
                *reinterpret_cast<u32x4*>(a.k_out + at) =
                    read_key<FMT, D>(a.cache, reinterpret_cast<const uint8_t*>(a.cache.k_pool) + page_head * IMAGE, page_head, slot, c);
        }
        __syncthreads();
        if (mine < n_heads && wanted) *reinterpret_cast<u32x4*>(a.v_out + at) = *reinterpret_cast<const u32x4*>(&s_v[turn][sub][slot][8 * c]);
    }
}

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
    const int64_t dense = int64_t(c.n_kv_heads) * c.head_dim;
    if (k_stride < dense || v_stride < dense) return fail(ST_ERR_SHAPE, "%s: a token stride of %lld elements for %d heads of %d", who, (long long)std::min(k_stride, v_stride), c.n_kv_heads, c.head_dim);
    if (k_stride % 8 != 0 || v_stride % 8 != 0) return fail(ST_ERR_INVALID_ARG, "%s: token strides must be multiples of 16 bytes", who);
    const int64_t capacity = int64_t(c.max_pages_per_seq) * kPage;
    if (host_len_upper_bound < 0 || host_len_upper_bound > capacity)
        return fail(ST_ERR_CAPACITY, "%s: length bound %d exceeds the page table (%lld tokens per sequence)", who, host_len_upper_bound, (long long)capacity);
    if (!aligned16(k_weight)) return fail(ST_ERR_INVALID_ARG, "%s: k_weight must be 16-byte aligned", who);
    if (!(eps >= 0.0)) return fail(ST_ERR_INVALID_ARG, "%s: eps must not be negative", who);
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
    a.touched = (max_n - 2 + kPage) / kPage + 1;
    const int64_t pages = int64_t(batch) * a.touched;
    const int hkv = c.n_kv_heads;
    a.head_groups = int(std::min<int64_t>(hkv, std::max<int64_t>(1, 2048 / pages)));
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
