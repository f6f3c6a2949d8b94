// Decode over 4-bit caches (ST_MXFP4: E2M1 codes, one power of two per 32 dims of a token): the split kernel of
// st_decode.hip's scheme -- work units, partial results, the same merge -- and a form that finishes short caches in one launch.
//
// HBM-bound in earnest: a token and KV head are D + D / 16 * 2 ... 136 bytes at D = 128, against 4 D G flops, so a compute unit gets one 16-token
// page of a head every 220 cycles at 6 TB/s and everything between the load and the matrix instruction has to fit into that.  The codes are laid out as
// the matrix instructions want them (st_kv_cache), one 16-byte load per lane, page and tensor:
//   K: lane (m = slot, g) holds 32 consecutive dims of its token -- one block, one scale.  The k-steps of the product take its four dwords in turn;
//      the query fragments use the same assignment of dims.
//   V: lane (m = dim % 16, g) holds slots 4 g .. + 3 of the D / 16 dims 16 j + m, which is what the score accumulator of lane group g holds
//      weights for: the weights go from one product into the other without an exchange.  A byte is dims d and d + 16 of ONE token, so one
//      conversion takes one scale.
// Codes become bf16 in registers, times their scale: exact (one bit of significand, powers of two).
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

template <int W, typename T>
__device__ __forceinline__ void load_words(uint32_t (&dst)[W], const T* p) {
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
    __device__ __forceinline__ void load(int s, int page, const uint8_t* kp, const uint8_t* vp, const uint8_t* sp, int n_kv_heads, Codes<D>& c) const {
        const int lane = int(threadIdx.x) & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t id = __builtin_amdgcn_readlane(page, 4 * s + u);
            const uint8_t* k_of = kp + id * n_kv_heads * (D * 8);
            const uint8_t* v_of = vp + id * n_kv_heads * (D * 8);
            const uint8_t* s_of = sp + id * n_kv_heads * D;
            // (64 dims: two lane groups share a block of 32, half of it each)
            load_words(c.k[u], k_of + (D == 128 ? lane * 16 : (g >> 1) * 256 + n * 16 + (g & 1) * 8));
            load_words(c.v[u], v_of + lane * (D / 8));
            c.ks[u] = s_of[D == 128 ? lane : (g >> 1) * 16 + n];
            load_words(c.vs[u], s_of + D / 2 + g * (D / 8));
        }
    }
    __device__ __forceinline__ void load(int s, int n_kv_heads, Codes<D>& c) const { load(s, my_page, k_pool, v_pool, scales, n_kv_heads, c); }
};

// bytes `i` of a scale word as the fp32 power of two
__device__ __forceinline__ float scale_of(uint32_t w, int i) { return __uint_as_float(((w >> (8 * i)) & 0xffu) << 23); }

__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float scale, int byte) {
    // (the byte is an immediate of the instruction)
    switch (byte) {
        case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
        case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
        case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
        default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
}

// Running state of 16 RB query rows, row 16 rb + n in the lanes (n, g), in base-2 exponent units.  The reference exponent of a row is the
// largest score so far (the weight of the row's largest score is 1, which rounds to itself), the sum takes the weights before they are rounded.
template <int D, int RB>
struct State4 {
    static constexpr int KS = D / 32, DB = D / 16, G = D / 32;
    bf16x8 qf[RB][KS];
    f32x4 o[RB][DB];
    float m[RB], l[RB];
    __device__ __forceinline__ State4() {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[r][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // largest of the four lanes n, n + 16, n + 32, n + 48 of a row
    static __device__ __forceinline__ float column_max(float x) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
        return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    // 64 tokens from token `tok` of a cache of `len` visible tokens, of which this lane's row rb sees [0, limit[rb]) and every row [0, limit_min)
    __device__ __forceinline__ void step(Codes<D>& c, int tok, int len, const int (&limit)[RB], int limit_min, float scale_log2) {
        const int g = int(threadIdx.x & 63) >> 4;
        f32x4 s[RB][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float ks = scale_of(c.ks[u], 0);
#pragma unroll
            for (int r = 0; r < RB; ++r) s[r][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                u32x4 kf;
#pragma unroll
                for (int i = 0; i < 4; ++i) kf[i] = fp4_pair(c.k[u][j], ks, i);
#pragma unroll
                for (int r = 0; r < RB; ++r) s[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), qf[r][j], s[r][u], 0, 0, 0);
            }
        }
        // register i of page u: token tok + 16 u + 4 g + i
        const int first = tok + 4 * g;
        const bool whole = tok + 64 <= limit_min;                        // uniform
        bf16x8 pb[RB][2];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = s[r][u][i] * scale_log2;
                    if (!whole) x = first + 16 * u + i < limit[r] ? x : -INFINITY;
                    s[r][u][i] = x;
                    mx = fmaxf(mx, x);
                }
            if (__any(mx > m[r])) {
                const float top = fmaxf(column_max(mx), m[r]);
                const float alpha = top > -INFINITY ? __builtin_amdgcn_exp2f(m[r] - top) : 1.f;
                m[r] = top;
                l[r] *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[r][db][i] *= alpha;
            }
            const float ref = m[r] > -INFINITY ? m[r] : 0.f;             // (nothing seen so far, or NaN alone)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(s[r][u][i] - ref);
                    l[r] += p;
                    pb[r][u >> 1][4 * (u & 1) + i] = (__bf16)p;
                }
        }
        if (tok + 64 > len) {
            // slots past the visible length hold anything: their weights are 0, their scales must be finite
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t keep = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) keep |= first + 16 * u + i < len ? 0xffu << (8 * i) : 0u;
#pragma unroll
                for (int gg = 0; gg < G; ++gg) c.vs[u][gg] &= keep;
            }
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int gg = 0; gg < G; ++gg) {
                // eight tokens (four of page 2 hf, four of the next), dims 32 gg + m and 32 gg + 16 + m
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = fp4_pair(c.v[2 * hf + (e >> 2)][gg], scale_of(c.vs[2 * hf + (e >> 2)][gg], e & 3), e & 3);
                u32x4 lo, hi;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100);
                    hi[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302);
                }
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    o[r][2 * gg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pb[r][hf], o[r][2 * gg], 0, 0, 0);
                    o[r][2 * gg + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pb[r][hf], o[r][2 * gg + 1], 0, 0, 0);
                }
            }
    }
};

// The queries of (sequence b, KV head h): row 16 rb + n is token row / G, head row % G; rows past the end repeat the last one (never stored).
// Fragment j holds dims dim0(g) + 8 j + e.  a.rope: rotated by the row's position, out of the table of the q_len positions.
template <int D, int RB>
__device__ __forceinline__ void load_queries(State4<D, RB>& st, const DecodeArgs& a, int b, int h, const float2* s_rot) {
    constexpr int KS = D / 32;
    const int lane = int(threadIdx.x) & 63, n = lane & 15, g = lane >> 4, dim0 = (D / 4) * g;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int row = min(16 * r + n, a.rows - 1), t = row / a.group;
        const uint16_t* qp = a.q + ((int64_t(b) * a.q_len + t) * a.n_q_heads + h * a.group + (row - t * a.group)) * D;
        const bool upper = dim0 >= D / 2;
        const int other0 = upper ? dim0 - D / 2 : dim0 + D / 2;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            bf16x8 x = *reinterpret_cast<const bf16x8*>(qp + dim0 + 8 * j);
            if (a.rope) {
                const bf16x8 y = *reinterpret_cast<const bf16x8*>(qp + other0 + 8 * j);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 cs = s_rot[t * (D / 2) + (upper ? other0 : dim0) + 8 * j + e];
                    const float own = float(x[e]), part = float(y[e]);
                    x[e] = (__bf16)(upper ? own * cs.x + part * cs.y : own * cs.x - part * cs.y);
                }
            }
            st.qf[r][j] = x;
        }
    }
}

// Row limits of a step over a cache: reasoning token j is seen by query token t where j <= len - q_len + t, the source slice by all
template <int RB>
__device__ __forceinline__ void row_limits(int (&limit)[RB], const DecodeArgs& a, bool is_src, int len) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int t = min(16 * r + (int(threadIdx.x) & 15), a.rows - 1) / a.group;
        limit[r] = is_src ? len : min(max(len - a.q_len + t + 1, 0), len);
    }
}

template <int D, int RB>
__global__ __launch_bounds__(64 * kSplitWaves, 2) void decode4_split_kernel(DecodeArgs a) {
    constexpr int DB = D / 16;
    // (cos, sin) of the q_len query positions; after the loop: SplitLds
    extern __shared__ __align__(16) unsigned char smem_raw[];
    float2* s_rot = reinterpret_cast<float2*>(smem_raw);
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
    int limit[RB];
    row_limits<RB>(limit, a, is_src, len);
    const int limit_min = is_src ? len : min(max(len - a.q_len + 1, 0), len);
    State4<D, RB> st;
    if (a.rope) {
        const int len_r = min(max(a.rsn_len[b], 0), a.rsn.max_pages * kPage);
        rope_table_to_lds<D>(s_rot, len_r - a.q_len, a.q_len, rope_frequency<D>(a.freq), 64 * kSplitWaves);
        lds_barrier();
    }
    load_queries<D, RB>(st, a, b, h, s_rot);
    for (int s = 0; s < n_steps; ++s) {
        Codes<D> codes;
        pages.load(s, a.n_kv_heads, codes);
        st.step(codes, unit0 + 64 * (wave + kSplitWaves * s), len, limit, limit_min, a.scale_log2);
    }
    __syncthreads();                                    // everybody is done with the rotations
    const SplitLds<D> sm(smem_raw, a.rows);
    const int n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        float l = st.l[r] + __shfl_xor(st.l[r], 16);
        l += __shfl_xor(l, 32);
        const int row = 16 * r + n;
        if (row < a.rows) {
            // lane (n, g), block db, register i  <->  d = 16 db + 4 g + i
            float* po = sm.o + (wave * a.rows + row) * D;
#pragma unroll
            for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(po + 16 * db + 4 * g) = st.o[r][db];
            if (g == 0) {
                sm.m[wave * a.rows + row] = st.m[r];
                sm.l[wave * a.rows + row] = l;
            }
        }
    }
    __syncthreads();
    merge_waves<D>(sm, a, ((int64_t(b) * a.n_kv_heads + h) * nc + c) * a.rows);
}

// Short caches: a workgroup of eight waves takes all of a (sequence, KV head) and finishes its rows -- one launch, no partial results.  Steps are
// dealt out as in the bf16 kernel: reasoning steps from the first wave up, source steps from the last one down.
constexpr int kSmallWaves4 = 8;

template <int D>
__global__ __launch_bounds__(64 * kSmallWaves4, 2) void decode4_small_kernel(DecodeArgs a, uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int DB = D / 16, W = kSmallWaves4;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    float* sm_o = reinterpret_cast<float*>(smem_raw);
    float2* sm_ml = reinterpret_cast<float2*>(sm_o + W * a.rows * D);
    float2* sm_rot = sm_ml + W * a.rows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = int(blockIdx.x % unsigned(a.n_kv_heads)), b = int(blockIdx.x / unsigned(a.n_kv_heads));
    const Pages4<D> pages_s(a.src, b, h, lane, 64 * (W - 1 - wave), W), pages_r(a.rsn, b, h, lane, 64 * wave, W);
    const int len_s = min(max(a.src_len[b], 0), a.src.max_pages * kPage), len_r = min(max(a.rsn_len[b], 0), a.rsn.max_pages * kPage);
    const int steps_s = (len_s - 64 * (W - 1 - wave) + 64 * W - 1) / (64 * W), steps_r = (len_r - 64 * wave + 64 * W - 1) / (64 * W);
    int limit_s[1], limit_r[1];
    row_limits<1>(limit_s, a, true, len_s);
    row_limits<1>(limit_r, a, false, len_r);
    const int limit_min = min(max(len_r - a.q_len + 1, 0), len_r);
    State4<D, 1> st;
    if (a.rope) {
        rope_table_to_lds<D>(sm_rot, len_r - a.q_len, a.q_len, rope_frequency<D>(a.freq), 64 * W);
        lds_barrier();
    }
    load_queries<D, 1>(st, a, b, h, sm_rot);
    for (int x = 0; x < steps_r + steps_s; ++x) {
        const bool r = x < steps_r;
        const int s = r ? x : x - steps_r;
        Codes<D> codes;
        pages_r.load(s, r ? pages_r.my_page : pages_s.my_page, r ? pages_r.k_pool : pages_s.k_pool, r ? pages_r.v_pool : pages_s.v_pool,
                     r ? pages_r.scales : pages_s.scales, a.n_kv_heads, codes);
        const int limit[1] = {r ? limit_r[0] : limit_s[0]};
        st.step(codes, 64 * ((r ? wave : W - 1 - wave) + W * s), r ? len_r : len_s, limit, r ? limit_min : len_s, a.scale_log2);
    }
    float l = st.l[0] + __shfl_xor(st.l[0], 16);
    l += __shfl_xor(l, 32);
    const int n = lane & 15, g = lane >> 4;
    if (n < a.rows) {
        float* po = sm_o + (wave * a.rows + n) * D;
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(po + 16 * db + 4 * g) = st.o[0][db];
        if (g == 0) sm_ml[wave * a.rows + n] = float2{st.m[0], l};
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
    const size_t rot = size_t(a.q_len) * (head_dim / 2) * sizeof(float2), smem = std::max(rot, split_lds_bytes(a.rows, head_dim));
    auto go = [&](auto kernel) -> st_status {
        const st_status r = allow_lds(kernel, smem);
        if (r == ST_OK) hipLaunchKernelGGL(kernel, dim3((unsigned)units), dim3(64 * kSplitWaves), smem, s, a);
        return r;
    };
    if (a.rows <= 16) return head_dim == 64 ? go(decode4_split_kernel<64, 1>) : go(decode4_split_kernel<128, 1>);
    return head_dim == 64 ? go(decode4_split_kernel<64, 2>) : go(decode4_split_kernel<128, 2>);
}

st_status launch_decode4_small(const DecodeArgs& a, int head_dim, uint16_t* out, float* lse, hipStream_t s) {
    const size_t smem = (size_t(kSmallWaves4) * a.rows * (head_dim + 2) + size_t(a.q_len) * head_dim) * sizeof(float);
    auto go = [&](auto kernel) -> st_status {
        const st_status r = allow_lds(kernel, smem);
        if (r == ST_OK) hipLaunchKernelGGL(kernel, dim3((unsigned)(a.batch * a.n_kv_heads)), dim3(64 * kSmallWaves4), smem, s, a, out, lse);
        return r;
    };
    return head_dim == 64 ? go(decode4_small_kernel<64>) : go(decode4_small_kernel<128>);
}

}  // namespace st
