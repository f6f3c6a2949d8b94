// Queries and keys normalised per head and rotated in one pass, and the gradients of that pass.
//
// A row x (one token of one head, D = 64 or 128 dims), weight w:
//   r = (mean x^2 + eps)^(-1/2),  n = x r w,  y = a R n
// with R the rotation of the row's leading `rot` dims by the token's position (a = 1 for dims past them).  Backwards, with
// g = dL/dy:  h = a R^T g,  dx = r (h w) - x r^3 / D * sum(h w x),  dw = sum over rows of h x r.
//
// Bound by HBM: forward 2 values moved per value, backward 3, some 10 and 25 operations each.  A row lies in D / 8
// neighbouring lanes, eight dims each, so that every access is 16 bytes per lane and whole lines per wave, and the sums over
// a row are data-parallel moves.  The (cos, sin) of a workgroup's tokens are evaluated once into LDS: one evaluation serves all heads.
// Measured, bf16, heads of 128 dims: forward of 131,072 tokens of 32 + 8 heads 495 us, 5.4 TB/s, what a copy reaches; of one token 3.4 us, a launch;
// backward of 16,001 tokens of 16 + 8 heads 59 us (5.0 TB/s) and 4.5 for the sum of the weights' gradients.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "st_norm.h"

namespace st {

st_status make_rope_table(const char* who, const st_rope_spec* spec, int head_dim, RopeTable* table) {
    if (!spec) return fail(ST_ERR_INVALID_ARG, "%s: rope spec is null", who);
    if (head_dim != 64 && head_dim != 128) return fail(ST_ERR_UNSUPPORTED, "%s: head_dim %d (64 or 128)", who, head_dim);
    // (64 pow calls are a good part of a short call's host time, and a program uses one spec: each thread keeps its last table)
    static thread_local RopeTable kept;
    static thread_local st_rope_spec kept_spec;
    static thread_local int kept_dim = 0;
    if (kept_dim == head_dim && memcmp(&kept_spec, spec, sizeof(kept_spec)) == 0) {
        *table = kept;
        return ST_OK;
    }
    const st_rope_spec& s = *spec;
    const int rot = s.rotary_dim == 0 ? head_dim : s.rotary_dim;
    auto positive = [](double x) { return x > 0.0 && x < HUGE_VAL; };
    if (!positive(s.theta_base)) return fail(ST_ERR_INVALID_ARG, "%s: theta_base must be positive", who);
    if (s.layout != ST_ROPE_HALF && s.layout != ST_ROPE_INTERLEAVED) return fail(ST_ERR_INVALID_ARG, "%s: rope layout %d", who, s.layout);
    if (s.rotary_dim < 0 || rot > head_dim) return fail(ST_ERR_SHAPE, "%s: rotary_dim %d of head_dim %d", who, s.rotary_dim, head_dim);
    if (rot % 16 != 0) return fail(ST_ERR_UNSUPPORTED, "%s: rotary_dim %d (a multiple of 16)", who, rot);
    if (s.scaling < ST_ROPE_PLAIN || s.scaling > ST_ROPE_YARN) return fail(ST_ERR_INVALID_ARG, "%s: rope scaling %d", who, s.scaling);
    if (s.scaling != ST_ROPE_PLAIN && !(s.factor >= 1.0 && s.factor < HUGE_VAL)) return fail(ST_ERR_INVALID_ARG, "%s: rope factor must be 1 or more", who);
    if (!(s.attention_factor >= 0.0 && s.attention_factor < HUGE_VAL)) return fail(ST_ERR_INVALID_ARG, "%s: attention_factor must be positive, or 0 for the default", who);
    double base = s.theta_base, lo = 0.0, hi = 0.0, a = 1.0;
    if (s.scaling == ST_ROPE_NTK) base *= pow(s.factor, double(rot) / double(rot - 2));
    if (s.scaling == ST_ROPE_YARN) {
        if (s.original_positions <= 0) return fail(ST_ERR_INVALID_ARG, "%s: original_positions must be positive", who);
        const double fast = s.beta_fast == 0.0 ? 32.0 : s.beta_fast, slow = s.beta_slow == 0.0 ? 1.0 : s.beta_slow;
        if (!positive(fast) || !positive(slow) || fast < slow) return fail(ST_ERR_INVALID_ARG, "%s: beta_fast / beta_slow", who);
        if (s.theta_base == 1.0) return fail(ST_ERR_INVALID_ARG, "%s: theta_base 1 has no turning frequencies", who);
        // the (real) pair index that turns `turns` times over the trained positions
        auto pair = [&](double turns) { return rot * log(s.original_positions / (turns * 6.283185307179586)) / (2.0 * log(s.theta_base)); };
        lo = std::max(floor(pair(fast)), 0.0);
        hi = std::min(ceil(pair(slow)), double(rot - 1));
        a = s.factor > 1.0 ? 0.1 * log(s.factor) + 1.0 : 1.0;
    }
    if (s.attention_factor > 0.0) a = s.attention_factor;
    RopeTable t;
    for (int i = 0; i < 64; ++i) {
        double f = i < rot / 2 ? pow(base, -2.0 * double(i) / double(rot)) : 0.0;
        if (s.scaling == ST_ROPE_LINEAR) f /= s.factor;
        if (s.scaling == ST_ROPE_YARN) {
            const double share = std::min(std::max((i - lo) / std::max(hi - lo, 1e-3), 0.0), 1.0);
            f = f * (1.0 - share) + f / s.factor * share;
        }
        t.f[i] = f;
    }
    t.rot = rot;
    t.interleaved = s.layout == ST_ROPE_INTERLEAVED;
    t.a = a;
    kept = t;
    kept_spec = s;
    kept_dim = head_dim;
    *table = t;
    return ST_OK;
}

// ---- eight dims of a row in a lane -------------------------------------------------------------------------------
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4 raw;
    __device__ __forceinline__ void load(const uint16_t* p) { raw = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(raw[i] << 16);
            f[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float (&f)[8]) {
        bf16x8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (__bf16)f[i];
        *reinterpret_cast<bf16x8*>(p) = r;
    }
};
template <>
struct Eight<float> {
    f32x4 lo, hi;
    __device__ __forceinline__ void load(const float* p) {
        lo = *reinterpret_cast<const f32x4*>(p);
        hi = *reinterpret_cast<const f32x4*>(p + 4);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = lo[i];
            f[4 + i] = hi[i];
        }
    }
    static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
        *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
    }
};

struct NormRows {                    // one of the two tensors, queries or keys
    void* out;                       // forward: y, dense; backward: dx
    const void* x;                   // NULL in a backward pass without a weight
    const void* g;                   // backward: dL/dy, dense
    const void* w;                   // NULL: not normalised
    int64_t out_stride, x_stride;    // elements from a token to the next
    int heads;
};
struct NormArgs {
    NormRows t[2];
    const int32_t* positions;
    int64_t n_tokens;
    int tokens;                      // of a workgroup's step
    float eps;
    double eps64;                    // for rows that are scaled; half its exponent (far below any row's for eps = 0)
    int eps_half;
    float* part;                     // backward: [workgroups][2][D] sums for the weights' gradients, or null
    RopeTable rope;
};

constexpr int kNormThreads = 256;

// (cos, sin) times a of `count` tokens from tok0 on: s_cos[t * rot / 2 + i], s_sin likewise.  The angle is reduced to an eighth of a turn in 64 bits:
// rounded to 32 at up to half a turn it would be off by 1.2e-7 (fp32 rows 7.3e-8 of their norm away from 64 bits; so 6.2e-8).
__device__ __forceinline__ void norm_table(const NormArgs& a, int64_t tok0, int count, float* s_cos, float* s_sin) {
    const int half = a.rope.rot / 2;
    for (int w = int(threadIdx.x); w < count * half; w += kNormThreads) {
        const int t = w / half, i = w - t * half;
        const double rev = double(a.positions[tok0 + t]) * a.rope.f[i] * 0.15915494309189535;        // angle / 2 pi
        const double turn = rev - rint(rev), quarter = rint(4.0 * turn);
        const int n = int(quarter) & 3;
        float sn, cs;
        sincosf(float((turn - 0.25 * quarter) * 6.283185307179586), &sn, &cs);
        const float c = n & 1 ? sn : cs, s = n & 1 ? cs : sn, f = float(a.rope.a);
        s_cos[w] = (n == 1 || n == 2 ? -c : c) * f;
        s_sin[w] = (n >= 2 ? -s : s) * f;
    }
}

// The lane's place in a rotation, and which sign its partners' share has.
template <int D>
struct Turn : RowTurn {
    float sign;
    bool interleaved;
    __device__ __forceinline__ Turn(const RopeTable& rope) : RowTurn(rope, int(threadIdx.x) % (D / 8)) {
        interleaved = rope.interleaved != 0;
        sign = high ? 1.f : -1.f;
    }
    // x turned by the token's angles (BACK: by their negatives); cos, sin: the token's row of the table
    template <bool BACK>
    __device__ __forceinline__ void apply(float (&x)[8], const float* cos, const float* sin) const {
        if (interleaved) {
            if (!turned) return;
            const f32x4 c = *reinterpret_cast<const f32x4*>(cos + at), s = *reinterpret_cast<const f32x4*>(sin + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = x[2 * i], hi = x[2 * i + 1], sn = BACK ? -s[i] : s[i];
                x[2 * i] = lo * c[i] - hi * sn;
                x[2 * i + 1] = hi * c[i] + lo * sn;
            }
            return;
        }
        float other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl(x[i], partner);
        if (!turned) return;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const f32x4 c = *reinterpret_cast<const f32x4*>(cos + at + 4 * u), s = *reinterpret_cast<const f32x4*>(sin + at + 4 * u);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * u + i] = x[4 * u + i] * c[i] + other[4 * u + i] * ((BACK ? -sign : sign) * s[i]);
        }
    }
};

// Whether a row's mean square, eps added, leaves it to 32 bits: no square, product or root of a row of this size is lost or overflows.  Other rows -- none
// where eps is one that models use -- are scaled by a power of two, eps with them: the norm of x 2^-e under eps 2^-2e is the norm of x.
__device__ __forceinline__ bool ordinary(float mean) { return mean > 0x1p-60f && mean < 0x1p80f; }
constexpr int kNoSize = -4096;
// The row's eight dims in a lane times 2^-e, e the exponent of the row's largest or of eps's root; the mean square of those.
template <int L>
__device__ __forceinline__ int scale_row(float (&x)[8], const NormArgs& a, float& mean) {
    float top = 0.f, ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
#pragma unroll
    for (int o = 1; o < L; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    int e = max(top > 0.f ? __builtin_amdgcn_frexp_expf(top) : kNoSize, a.eps_half);
    e = e == kNoSize || top == INFINITY ? 0 : e;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = ldexpf(x[i], -e);
        ss = fmaf(x[i], x[i], ss);
    }
    mean = row_sum<L>(ss) * (1.f / (8 * L)) + float(ldexp(a.eps64, -2 * e));
    return e;
}

// Forward.  A workgroup takes rows [block * rows, + rows) of the n_tokens * (q_heads + k_heads) rows of both tensors, token by
// token: few rows (down to one pass) where there are few in all, so that a decoding step's token is one memory round trip.  The next
// pass's rows are asked for before this one's are worked on.
template <typename T, int D>
__global__ __launch_bounds__(kNormThreads) void norm_rope_kernel(NormArgs a, int rows) {
    constexpr int L = D / 8, RP = kNormThreads / L;
    extern __shared__ __align__(16) float smem[];
    const int heads = a.t[0].heads + a.t[1].heads, half = a.rope.rot / 2;
    const int64_t row0 = int64_t(blockIdx.x) * rows, n_rows = a.n_tokens * heads;
    const int64_t tok0 = row0 / heads;
    const int count = int(min(int64_t(rows), n_rows - row0));
    const int first = int(row0 - tok0 * heads);                      // row of token tok0 that the workgroup begins with
    const int n_tok = (first + count - 1) / heads + 1;
    float *s_cos = smem, *s_sin = smem + a.tokens * half;
    const int c = int(threadIdx.x) % L;
    auto place = [&](int r, int& tok, int& h) {
        tok = (first + r) / heads;
        h = first + r - tok * heads;
    };
    auto load = [&](int tok, int h, Eight<T>& e) {
        const bool second = h >= a.t[0].heads;
        const T* src = static_cast<const T*>(second ? a.t[1].x : a.t[0].x) + (tok0 + tok) * (second ? a.t[1].x_stride : a.t[0].x_stride);
        e.load(src + (second ? h - a.t[0].heads : h) * D + 8 * c);
    };
    Eight<T> next;
    int r = int(threadIdx.x) / L, tok, h;
    place(r, tok, h);
    if (r < count) load(tok, h, next);
    Eight<T> w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (a.t[i].w) w[i].load(static_cast<const T*>(a.t[i].w) + 8 * c);
    norm_table(a, tok0, n_tok, s_cos, s_sin);
    const Turn<D> turn(a.rope);
    __syncthreads();
    // (all lanes of a row are in or out together)
    while (r < count) {
        const Eight<T> now = next;
        const int t_now = tok, h_now = h;
        r += RP;
        if (r < count) {
            h += RP;
            while (h >= heads) {
                h -= heads;
                ++tok;
            }
            load(tok, h, next);
        }
        float x[8];
        now.get(x);
        const bool second = h_now >= a.t[0].heads;
        if (second ? a.t[1].w != nullptr : a.t[0].w != nullptr) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
            float mean = row_sum<L>(ss) * (1.f / D) + a.eps;
            if (!ordinary(mean)) scale_row<L>(x, a, mean);
            const float rs = rsqrtf(mean);
            float w0[8], w1[8];
            w[0].get(w0);
            w[1].get(w1);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * rs * (second ? w1[i] : w0[i]);
        }
        turn.template apply<false>(x, s_cos + t_now * half, s_sin + t_now * half);
        T* dst = static_cast<T*>(second ? a.t[1].out : a.t[0].out) + (tok0 + t_now) * (second ? a.t[1].out_stride : a.t[0].out_stride);
        Eight<T>::store(dst + (second ? h_now - a.t[0].heads : h_now) * D + 8 * c, x);
    }
}

// Backward.  Workgroups walk steps of a.tokens tokens, first the query rows of a step, then its key rows, and keep the sums for the
// weights' gradients in registers; each leaves one partial sum per tensor, added up in a fixed order by weight_sum_kernel.
// (A step's first rows asked for before its table: bf16 1 % faster, fp32 40 % slower, for want of registers.  The four workgroups per compute unit are asked
// for: fp32 rows take 128 registers and a few spilled ones, with 130 1,801 tokens of 24 heads were 24.8 us instead of 22 before the sums below took their present form.)
template <typename T, int D>
__global__ __launch_bounds__(kNormThreads, 4) void norm_rope_bwd_kernel(NormArgs a) {
    constexpr int L = D / 8, RP = kNormThreads / L;
    extern __shared__ __align__(16) float smem[];
    const int half = a.rope.rot / 2, c = int(threadIdx.x) % L, row = int(threadIdx.x) / L;
    float *s_cos = smem, *s_sin = smem + a.tokens * half;
    const Turn<D> turn(a.rope);
    float dw[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.f;

    auto walk = [&](int64_t tok0, int n_tok, auto which) {
        constexpr int W = decltype(which)::value;
        const NormRows& t = a.t[W];
        if (t.heads == 0) return;
        float w[8];
        if (t.w) {
            Eight<T> e;
            e.load(static_cast<const T*>(t.w) + 8 * c);
            e.get(w);
        }
        const int count = n_tok * t.heads;
        int tok = row / t.heads, h = row - tok * t.heads;
        auto load = [&](Eight<T>& g, Eight<T>& x) {
            g.load(static_cast<const T*>(t.g) + ((tok0 + tok) * t.heads + h) * D + 8 * c);
            if (t.w) x.load(static_cast<const T*>(t.x) + (tok0 + tok) * t.x_stride + h * D + 8 * c);
        };
        Eight<T> g_next, x_next;
        int r = row;
        if (r < count) load(g_next, x_next);
        while (r < count) {
            const Eight<T> g_now = g_next, x_now = x_next;
            const int t_now = tok, h_now = h;
            r += RP;
            if (r < count) {
                h += RP;
                while (h >= t.heads) {
                    h -= t.heads;
                    ++tok;
                }
                load(g_next, x_next);
            }
            float g[8];
            g_now.get(g);
            turn.template apply<true>(g, s_cos + t_now * half, s_sin + t_now * half);
            if (t.w) {
                float x[8], ss = 0.f, sg = 0.f;
                x_now.get(x);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    ss = fmaf(x[i], x[i], ss);
                    sg = fmaf(g[i] * w[i], x[i], sg);
                }
                float mean = row_sum<L>(ss) * (1.f / D) + a.eps;
                int e = 0;
                if (!ordinary(mean)) {
                    e = scale_row<L>(x, a, mean);
                    sg = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sg = fmaf(g[i] * w[i], x[i], sg);
                }
                const float rs = rsqrtf(mean);
                const float back = row_sum<L>(sg) * (1.f / D) * rs * rs;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xr = x[i] * rs;
                    dw[W][i] = fmaf(g[i], xr, dw[W][i]);
                    g[i] = rs * (g[i] * w[i] - x[i] * back);
                }
                if (e != 0)
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = ldexpf(g[i], -e);
            }
            Eight<T>::store(static_cast<T*>(t.out) + (tok0 + t_now) * t.out_stride + h_now * D + 8 * c, g);
        }
    };
    for (int64_t tok0 = int64_t(blockIdx.x) * a.tokens; tok0 < a.n_tokens; tok0 += int64_t(gridDim.x) * a.tokens) {
        const int n_tok = int(min(int64_t(a.tokens), a.n_tokens - tok0));
        norm_table(a, tok0, n_tok, s_cos, s_sin);
        __syncthreads();
        walk(tok0, n_tok, std::integral_constant<int, 0>{});
        walk(tok0, n_tok, std::integral_constant<int, 1>{});
        __syncthreads();
    }
    if (!a.part) return;
    // the sums of the workgroup's rows over its lane groups, in a fixed order and in 64 bits: a lane has a few rows in 32, and what comes after them adds nothing but the
    // rounding of the partial sum (16,001 tokens of 24 bf16 heads: gradients 8.8e-8 of their norm from the definition, with shuffles and sums in 32 bits
    // 10.0e-8; 1,801 tokens in fp32: 7.4e-8 and 8.8e-8, 20.6 and 21.7 us)
    float* s_dw = smem;                                    // [RP][2][D]
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
            *reinterpret_cast<f32x4*>(s_dw + (row * 2 + t) * D + 8 * c + 4 * u) = f32x4{dw[t][4 * u], dw[t][4 * u + 1], dw[t][4 * u + 2], dw[t][4 * u + 3]};
    __syncthreads();
    for (int i = int(threadIdx.x); i < 2 * D; i += kNormThreads) {
        double v = 0.0;
#pragma unroll
        for (int u = 0; u < RP; ++u) v += double(s_dw[u * 2 * D + i]);
        a.part[int64_t(blockIdx.x) * (2 * D) + i] = float(v);
    }
}

// The workgroups' partial sums, 16 columns per workgroup: 64 groups of four lanes take every 64th row, in a fixed order.  In 64 bits, which costs nothing
// here: a thousand sums of either sign, added in 32, put as much error into the result as all the rows before.
__global__ __launch_bounds__(256) void weight_sum_kernel(const float* __restrict__ part, int n_part, int dim, float* __restrict__ dqw,
                                                         float* __restrict__ dkw) {
    typedef double f64x4 __attribute__((ext_vector_type(4)));
    __shared__ f64x4 s_sum[256];
    const int col = int(blockIdx.x) * 16 + 4 * (int(threadIdx.x) & 3);
    f64x4 sum = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
    for (int r = int(threadIdx.x) >> 2; r < n_part; r += 64) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(part + int64_t(r) * 2 * dim + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += double(x[e]);
    }
    s_sum[threadIdx.x] = sum;
    __syncthreads();
    for (int n = 128; n >= 4; n >>= 1) {
        if (int(threadIdx.x) < n) s_sum[threadIdx.x] += s_sum[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x < 4) {
        float* dst = col < dim ? dqw : dkw;
        if (dst)
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[col % dim + i] = float(s_sum[threadIdx.x][i]);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
// Tokens of a step and steps in flight of the backward pass: at most 1,024 workgroups (four per compute unit) that leave sums for the weights, and where
// there are tokens enough, as many in a step as make four passes of the workgroup's threads.  16,001 tokens of 24 heads of 128: 65 us, with 512 workgroups
// 76, with 2,048 69, with two tokens a step 66, with eight 68; 131,072 of 40: 752, with four tokens instead of two 778; 65,536 of 18 heads of 64: 96, with
// four instead of eight 106; 100,000 of 3 of 64: 42, with four instead of 32 94; 1,801 of 24 fp32 heads: 21, with 512 workgroups 20, with 2,048 25.
constexpr int kBwdWorkgroups = 1024;
inline int bwd_tokens(int64_t n_tokens, int64_t heads, int head_dim) {
    int tokens = 1;
    while (tokens < 32 && tokens * heads < 4 * kNormThreads / (head_dim / 8) && n_tokens >= 2 * tokens * kBwdWorkgroups) tokens *= 2;
    return tokens;
}
inline int bwd_workgroups(int64_t n_tokens, int64_t heads, int head_dim) {
    const int tokens = bwd_tokens(n_tokens, heads, head_dim);
    return int(std::min<int64_t>((n_tokens + tokens - 1) / tokens, kBwdWorkgroups));
}

inline void set_eps(NormArgs& a, double eps) {
    a.eps = float(eps);
    a.eps64 = eps;
    a.eps_half = eps > 0.0 ? (ilogb(eps) + 2) / 2 : kNoSize;
}
// What both directions ask of the sizes.  (Rows of a workgroup are counted in 32 bits, rows of a call in 64.)
static st_status check_sizes(const char* who, int64_t n_tokens, int n_q_heads, int n_kv_heads, double eps) {
    if (n_tokens < 0 || n_q_heads <= 0 || n_kv_heads < 0) return fail(ST_ERR_INVALID_ARG, "%s: bad sizes", who);
    if (n_q_heads > (1 << 16) || n_kv_heads > (1 << 16) || n_tokens > (int64_t(1) << 40)) return fail(ST_ERR_SHAPE, "%s: more than 65,536 heads or 2^40 tokens", who);
    if (!(eps >= 0.0 && eps < HUGE_VAL)) return fail(ST_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
    return ST_OK;
}
// what both directions ask of one tensor's arguments
static st_status check_rows(const char* who, const char* name, const void* p, const void* w, int64_t stride, int heads, int head_dim, size_t size) {
    if (!p) return fail(ST_ERR_INVALID_ARG, "%s: %s is null", who, name);
    if (!aligned16(p) || !aligned16(w)) return fail(ST_ERR_INVALID_ARG, "%s: %s and its weight must be 16-byte aligned", who, name);
    if (stride < int64_t(heads) * head_dim) return fail(ST_ERR_SHAPE, "%s: %s has a token stride of %lld elements for %d heads of %d", who, name, (long long)stride, heads, head_dim);
    if (stride * int64_t(size) % 16 != 0) return fail(ST_ERR_INVALID_ARG, "%s: %s needs a token stride of a multiple of 16 bytes", who, name);
    return ST_OK;
}

}  // namespace st

using namespace st;

extern "C" st_status st_norm_rope_apply_qk(void* q_out, const void* q, int64_t q_stride, int32_t n_q_heads, const void* q_weight, void* k_out,
                                           const void* k, int64_t k_stride, int32_t n_kv_heads, const void* k_weight,
                                           const int32_t* positions, int64_t n_tokens, int32_t head_dim, double eps,
                                           const st_rope_spec* spec, st_dtype dt, void* hip_stream) {
    const char* who = "st_norm_rope_apply_qk";
    if (dt != ST_F32 && dt != ST_BF16) return fail(ST_ERR_UNSUPPORTED, "%s: dtype %d", who, int(dt));
    const size_t size = dt == ST_F32 ? 4 : 2;
    NormArgs a{};
    st_status r = make_rope_table(who, spec, head_dim, &a.rope);
    if (r != ST_OK) return r;
    r = check_sizes(who, n_tokens, n_q_heads, n_kv_heads, eps);
    if (r != ST_OK) return r;
    if (n_tokens == 0) return ST_OK;
    if (!positions) return fail(ST_ERR_INVALID_ARG, "%s: positions is null", who);
    const struct { void* out; const void* x; int64_t stride; int heads; const void* w; const char* name; } in[2] = {
        {q_out, q, q_stride, n_q_heads, q_weight, "q"}, {k_out, k, k_stride, n_kv_heads, k_weight, "k"}};
    for (int i = 0; i < (n_kv_heads > 0 ? 2 : 1); ++i) {
        r = check_rows(who, in[i].name, in[i].x, in[i].w, in[i].stride, in[i].heads, head_dim, size);
        if (r != ST_OK) return r;
        if (!in[i].out || !aligned16(in[i].out)) return fail(ST_ERR_INVALID_ARG, "%s: %s_out must be non-null and 16-byte aligned", who, in[i].name);
        const int64_t dense = int64_t(in[i].heads) * head_dim;
        if (in[i].out == in[i].x && in[i].stride != dense) return fail(ST_ERR_INVALID_ARG, "%s: %s in place must be dense", who, in[i].name);
        a.t[i] = NormRows{in[i].out, in[i].x, nullptr, in[i].w, dense, in[i].stride, in[i].heads};
    }
    a.positions = positions;
    a.n_tokens = n_tokens;
    set_eps(a, eps);
    // Rows of a workgroup: one pass of its threads while that makes no more than 1,024 workgroups, else up to four tokens, whose table
    // the heads share.  131,072 tokens of 40 heads: 495 us, one token each 493, sixteen 539; 4,099 of 18 fp32 heads: 9.4 us, with up to 256
    // workgroups 9.5, up to 4,096 10.9, one token each 10.7.
    const int heads = n_q_heads + n_kv_heads, pass = kNormThreads / (head_dim / 8);
    const int64_t n_rows = n_tokens * heads;
    int rows = pass;
    while (rows < 4 * heads && (n_rows + rows - 1) / rows > 1024) rows += pass;
    const int64_t blocks = (n_rows + rows - 1) / rows;
    if (blocks > 0x7fffffff) return fail(ST_ERR_SHAPE, "%s: too many rows", who);
    a.tokens = (rows - 1 + heads - 1) / heads + 1;                 // tokens that `rows` rows may touch, wherever they begin
    const size_t smem = size_t(a.tokens) * a.rope.rot * sizeof(float);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kNormThreads), smem, s, a, rows); };
    if (dt == ST_F32) {
        if (head_dim == 64) go(norm_rope_kernel<float, 64>); else go(norm_rope_kernel<float, 128>);
    } else {
        if (head_dim == 64) go(norm_rope_kernel<uint16_t, 64>); else go(norm_rope_kernel<uint16_t, 128>);
    }
    ST_LAUNCH_CHECK("norm_rope_kernel");
    return ST_OK;
}

extern "C" size_t st_norm_rope_bwd_workspace_bytes(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_tokens < 0 || n_q_heads <= 0 || n_kv_heads < 0 || (head_dim != 64 && head_dim != 128)) return 0;
    return size_t(bwd_workgroups(n_tokens, int64_t(n_q_heads) + n_kv_heads, head_dim)) * 2 * head_dim * sizeof(float);
}

extern "C" st_status st_norm_rope_bwd_qk(void* dq, int64_t dq_stride, float* dq_weight, const void* d_q_out, const void* q, int64_t q_stride,
                                         int32_t n_q_heads, const void* q_weight, void* dk, int64_t dk_stride, float* dk_weight,
                                         const void* d_k_out, const void* k, int64_t k_stride, int32_t n_kv_heads, const void* k_weight,
                                         const int32_t* positions, int64_t n_tokens, int32_t head_dim, double eps,
                                         const st_rope_spec* spec, st_dtype dt, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "st_norm_rope_bwd_qk";
    if (dt != ST_F32 && dt != ST_BF16) return fail(ST_ERR_UNSUPPORTED, "%s: dtype %d", who, int(dt));
    const size_t size = dt == ST_F32 ? 4 : 2;
    NormArgs a{};
    st_status r = make_rope_table(who, spec, head_dim, &a.rope);
    if (r != ST_OK) return r;
    r = check_sizes(who, n_tokens, n_q_heads, n_kv_heads, eps);
    if (r != ST_OK) return r;
    if (!positions && n_tokens > 0) return fail(ST_ERR_INVALID_ARG, "%s: positions is null", who);
    const struct { void* dx; int64_t dx_stride; float* dw; const void* g; const void* x; int64_t x_stride; int heads; const void* w; const char *name, *dname; } in[2] = {
        {dq, dq_stride, dq_weight, d_q_out, q, q_stride, n_q_heads, q_weight, "q", "dq"},
        {dk, dk_stride, dk_weight, d_k_out, k, k_stride, n_kv_heads, k_weight, "k", "dk"}};
    bool sums = false;
    for (int i = 0; i < (n_kv_heads > 0 ? 2 : 1); ++i) {
        if (in[i].dw && !in[i].w) return fail(ST_ERR_INVALID_ARG, "%s: the gradient of a weight that is null", who);
        if (in[i].dw && (reinterpret_cast<uintptr_t>(in[i].dw) & 3u)) return fail(ST_ERR_INVALID_ARG, "%s: weight gradients must be 4-byte aligned", who);
        sums = sums || in[i].dw;
        if (n_tokens == 0) continue;
        r = check_rows(who, in[i].dname, in[i].dx, nullptr, in[i].dx_stride, in[i].heads, head_dim, size);
        if (r != ST_OK) return r;
        if (!in[i].g || !aligned16(in[i].g)) return fail(ST_ERR_INVALID_ARG, "%s: the gradient of %s's result must be non-null and 16-byte aligned", who, in[i].name);
        if (in[i].w) {
            r = check_rows(who, in[i].name, in[i].x, in[i].w, in[i].x_stride, in[i].heads, head_dim, size);
            if (r != ST_OK) return r;
            // a row is read as a whole before it is written, but only where it lies itself
            if (in[i].dx == in[i].x && in[i].dx_stride != in[i].x_stride) return fail(ST_ERR_INVALID_ARG, "%s: %s over %s needs the same strides", who, in[i].dname, in[i].name);
        }
        if (in[i].dx == in[i].g && in[i].dx_stride != int64_t(in[i].heads) * head_dim)
            return fail(ST_ERR_INVALID_ARG, "%s: %s over the gradient of its result must be dense", who, in[i].dname);
        a.t[i] = NormRows{in[i].dx, in[i].x, in[i].g, in[i].w, in[i].dx_stride, in[i].x_stride, in[i].heads};
    }
    if (n_kv_heads == 0 && dk_weight) return fail(ST_ERR_INVALID_ARG, "%s: the gradient of a weight that is null", who);
    if (sums && n_tokens > 0) {
        const size_t need = st_norm_rope_bwd_workspace_bytes(n_tokens, n_q_heads, n_kv_heads, head_dim);
        if (!workspace || !aligned16(workspace)) return fail(ST_ERR_INVALID_ARG, "%s: workspace must be non-null and 16-byte aligned", who);
        if (workspace_bytes < need) return fail(ST_ERR_CAPACITY, "%s: workspace has %zu bytes, needs %zu", who, workspace_bytes, need);
        a.part = static_cast<float*>(workspace);
    }
    if (dq_weight && dq_weight == dk_weight) return fail(ST_ERR_INVALID_ARG, "%s: dq_weight and dk_weight are one array", who);
    a.positions = positions;
    a.n_tokens = n_tokens;
    set_eps(a, eps);
    a.tokens = bwd_tokens(n_tokens, int64_t(n_q_heads) + n_kv_heads, head_dim);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int blocks = bwd_workgroups(n_tokens, int64_t(n_q_heads) + n_kv_heads, head_dim);
    if (blocks > 0) {
        const size_t smem = std::max(size_t(a.tokens) * a.rope.rot * sizeof(float), size_t(kNormThreads) * 2 * 8 * sizeof(float));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kNormThreads), smem, s, a); };
        if (dt == ST_F32) {
            if (head_dim == 64) go(norm_rope_bwd_kernel<float, 64>); else go(norm_rope_bwd_kernel<float, 128>);
        } else {
            if (head_dim == 64) go(norm_rope_bwd_kernel<uint16_t, 64>); else go(norm_rope_bwd_kernel<uint16_t, 128>);
        }
        ST_LAUNCH_CHECK("norm_rope_bwd_kernel");
    }
    if (sums) {
        // (no tokens: the sums are 0)
        hipLaunchKernelGGL(weight_sum_kernel, dim3((unsigned)(2 * head_dim / 16)), dim3(256), 0, s, static_cast<const float*>(a.part), blocks, head_dim, dq_weight, dk_weight);
        ST_LAUNCH_CHECK("weight_sum_kernel");
    }
    return ST_OK;
}
