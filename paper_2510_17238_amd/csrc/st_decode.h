// What the decode kernels of bf16, 8-bit and 4-bit caches share (internal).
#pragma once
#include <type_traits>

#include "st_cache.h"
#include "st_tiles.h"

namespace st {

struct DecodeArgs {
    CacheView src, rsn;
    const int32_t* src_len;
    const int32_t* rsn_len;
    const uint16_t* q;
    float* part_o;     // [B][Hkv][nc][rows][D]
    float* part_ml;    // [B][Hkv][nc][rows][2]
    int batch, q_len, n_q_heads, n_kv_heads, group, rows;
    int ncs, ncr;      // chunk slots per (sequence, head) for the two caches
    int chunk;         // tokens per work unit (kChunkMin .. kChunkLong)
    float scale_log2;
    // source-chunk prefill only: ragged query counts and 32-row blocks
    const int32_t* n_new;   // [B] query tokens per sequence, or null for max_new everywhere
    int max_new;            // token stride of q / out
    int row_blocks;         // ceil(max_new * group / 32)
    // fused query rotation: q holds unrotated queries; row t is the token at index len - q_len + t of its own
    // stream (reasoning for a decode step, source for a source chunk), which is its position id
    int rope;
    RopeFreq freq;
    // one decoding step in one call (bf16, q_len = 1, <= 16 rows): the token k_new / v_new [batch][Hkv][D] is the one at
    // index rsn_len[b] - 1 of the reasoning stream and is NOT in the cache yet -- the launch stores it, attends over
    // the cached tokens before it, and takes the token itself from registers as one more partial state
    int append;
    const uint16_t* k_new;
    const uint16_t* v_new;
    // wave timeline (st_profile_wave_trace): (start, end) wall-clock pairs per workgroup, or null
    unsigned long long* trace;
    int trace_cap;
};

// Stamps the workgroup's start and end into the timeline buffer, whichever way the kernel is left.
struct WaveStamp {
    unsigned long long* slot;
    unsigned long long t0;
    __device__ __forceinline__ WaveStamp(const DecodeArgs& a) : slot(nullptr), t0(0) {
        if (a.trace && int(blockIdx.x) < a.trace_cap) {
            slot = a.trace + 2 * size_t(blockIdx.x);
            t0 = wall_clock64();
        }
    }
    __device__ __forceinline__ ~WaveStamp() {
        if (slot && threadIdx.x == 0) {
            slot[0] = t0;
            slot[1] = wall_clock64();
        }
    }
};

// A barrier for data exchanged through LDS alone: __syncthreads() also waits for every global load in flight -- here the first
// keys and values, requested before the queries are rotated.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The split kernels: a workgroup of FOUR WAVES takes one work unit (one cache of one sequence and KV head, a.chunk tokens)
// and deals its steps out to the waves in turn; their states meet in LDS and ONE partial result leaves the
// workgroup.  A partial is rows x D floats, written and read back by the merge kernel: with a wave per unit either the units
// were short and the partials cost more than the bytes alone say (64 sequences of up to 24K tokens, 32 rows: 512-token units
// 910 us, 1,024-token units 852), or they were long and the launch ended with a few of them.
constexpr int kSplitWaves = 4;

// what the waves of a workgroup leave for the merge: [4][rows][D] un-normalised outputs, [4][rows] reference exponents and sums
template <int D>
struct SplitLds {
    float *o, *m, *l;
    __device__ __forceinline__ SplitLds(unsigned char* smem, int rows)
        : o(reinterpret_cast<float*>(smem)), m(o + kSplitWaves * rows * D), l(m + kSplitWaves * rows) {}
};
inline size_t split_lds_bytes(int rows, int d) { return sizeof(float) * size_t(kSplitWaves) * rows * (d + 2); }

// A state (reference exponent m, sum l) without a finite score: nothing that its row sees -- or NaN scores alone, whose sum says
// so and has to reach the row (its weight 2^(-inf) = 0 keeps a NaN one).
__device__ __forceinline__ bool holds_nothing(float m, float l) { return m == -INFINITY && l == 0.f; }

// log-sum-exp merge of the waves' states of `rows` rows into the unit's partial result at row slot `slot`
template <int D>
__device__ __forceinline__ void merge_waves(const SplitLds<D>& sm, const int& rows, const DecodeArgs& a, int64_t slot) {
    for (int e = int(threadIdx.x) * 4; e < rows * D; e += 64 * kSplitWaves * 4) {
        const int row = e / D, d0 = e % D;
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w) m_all = fmaxf(m_all, sm.m[w * rows + row]);
        const float m_use = m_all == -INFINITY ? 0.f : m_all;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w) {
            const float mw = sm.m[w * rows + row], lw = sm.l[w * rows + row];
            if (holds_nothing(mw, lw)) continue;
            const float wt = __builtin_amdgcn_exp2f(mw - m_use);
            den = fmaf(wt, lw, den);
            const f32x4 o = *reinterpret_cast<const f32x4*>(sm.o + (w * rows + row) * D + d0);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = fmaf(wt, o[i], acc[i]);
        }
        *reinterpret_cast<f32x4*>(a.part_o + (slot + row) * D + d0) = acc;
        if (d0 == 0) {
            a.part_ml[(slot + row) * 2] = m_all;
            a.part_ml[(slot + row) * 2 + 1] = den;
        }
    }
}

// Unit of a workgroup among the nc of its (sequence, KV head).  Consecutive workgroups go to the eight XCDs in turn: where nc shares a
// factor g with 8, the same unit of every head would land on the same 8 / g of them -- and with caches of unlike length it is the
// first units that have tokens (128 sequences of 300 + 300 tokens and one of 12,000, eight slots a head: 163 us, with 72 us of
// work; now 97).  So the units of a head are turned by one place whenever the heads have been once around the XCDs.
__device__ __forceinline__ int unit_of(unsigned block, int nc) {
    const unsigned bh = block / unsigned(nc), i = block % unsigned(nc), g = min(unsigned(nc & -nc), 8u);
    return int(g == 1 ? i : (i + bh * g / 8) % unsigned(nc));
}

// The states of a workgroup that holds ALL of its rows' tokens -- WP states, [WP][rows][D] un-normalised outputs and [WP][rows] (reference
// exponent, sum) in LDS, 64 W threads -- merged by log-sum-exp in a fixed order into the finished rows of (sequence b, KV head h).
template <int D, int W, int WP>
__device__ __forceinline__ void merge_and_store(const float* sm_o, const float2* sm_ml, const DecodeArgs& a, int b, int h, uint16_t* __restrict__ out, float* __restrict__ lse) {
    // Merge: a thread takes one dim of a row, two or four where the rows have more than the threads; everything it needs is read at once, and
    // all waves take part.  (State by state, each with a branch, by the threads that had four dims: 2,900 of the workgroup's 15,800 cycles
    // with 4 rows of 128 dims, now 2,000; 36 layers of one token, 32 / 8 heads, 400 cached tokens 298.5 -> 291.5 us.)
    auto merge = [&](auto width) {
        constexpr int N = decltype(width)::value;
        for (int e = int(threadIdx.x) * N; e < a.rows * D; e += 64 * W * N) {
            const int row = e / D, d0 = e % D;
            float mw[WP], lw[WP], o[WP][N], m_all = -INFINITY;
#pragma unroll
            for (int w = 0; w < WP; ++w) {
                const float2 ml = sm_ml[w * a.rows + row];
                mw[w] = ml.x;
                lw[w] = ml.y;
                const float* po = sm_o + (w * a.rows + row) * D + d0;
                if constexpr (N == 4) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(po);
#pragma unroll
                    for (int i = 0; i < N; ++i) o[w][i] = x[i];
                } else {
                    const f32x2 x = N == 2 ? *reinterpret_cast<const f32x2*>(po) : f32x2{po[0], 0.f};
#pragma unroll
                    for (int i = 0; i < N; ++i) o[w][i] = x[i];
                }
            }
#pragma unroll
            for (int w = 0; w < WP; ++w) m_all = fmaxf(m_all, mw[w]);
            float acc[N], den = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WP; ++w) {
                // (a state that holds nothing may hold anything in its output)
                const bool skip = m_all == -INFINITY || holds_nothing(mw[w], lw[w]);
                const float wt = skip ? 0.f : __builtin_amdgcn_exp2f(mw[w] - m_all);
                den = skip ? den : fmaf(wt, lw[w], den);
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = skip ? acc[i] : fmaf(wt, o[w][i], acc[i]);
            }
            const float inv = den > 0.f ? 1.f / den : 0.f;           // a row that sees nothing: out = 0, lse = -inf
            const int t = a.q_len == 1 ? 0 : row / a.group, hq_row = h * a.group + (row - t * a.group);
            uint16_t* dst = out + ((int64_t(b) * a.q_len + t) * a.n_q_heads + hq_row) * D + d0;
            if constexpr (N == 4) {
                bf16x4 o4;
#pragma unroll
                for (int i = 0; i < 4; ++i) o4[i] = (__bf16)(acc[i] * inv);
                *reinterpret_cast<bf16x4*>(dst) = o4;
            } else if constexpr (N == 2) {
                bf16x2 o2;
                o2[0] = (__bf16)(acc[0] * inv);
                o2[1] = (__bf16)(acc[1] * inv);
                *reinterpret_cast<bf16x2*>(dst) = o2;
            } else {
                *reinterpret_cast<__bf16*>(dst) = (__bf16)(acc[0] * inv);
            }
            if (lse && d0 == 0)
                lse[(int64_t(b) * a.q_len + t) * a.n_q_heads + hq_row] = den > 0.f ? (m_all + __builtin_amdgcn_logf(den)) * kLn2 : -INFINITY;
        }
    };
    if (a.rows * D <= 64 * W) merge(std::integral_constant<int, 1>{});
    else if (a.rows * D <= 64 * W * 2) merge(std::integral_constant<int, 2>{});
    else merge(std::integral_constant<int, 4>{});
}

// The split kernels over 4-bit caches (st_decode4.hip): the launch that leaves the partial results of a step, and the one
// that finishes short caches by itself.
st_status launch_decode4(const DecodeArgs& a, int head_dim, int64_t units, hipStream_t s);
st_status launch_decode4_small(const DecodeArgs& a, int head_dim, uint16_t* out, float* lse, hipStream_t s);

}  // namespace st
