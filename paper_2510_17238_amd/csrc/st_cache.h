// Kernel-side view of one paged KV cache (internal).
#pragma once
#include "st_internal.h"

namespace st {

struct CacheView {
    uint16_t* k_pool;            // [n_pages][Hkv][D/8][16][8] bf16 bits
    uint16_t* v_pool;            // [n_pages][Hkv][D][16]
    const int32_t* page_table;   // [batch][max_pages]
    int32_t* appended_len;       // [batch]
    int32_t max_pages;
    int32_t n_pages;
    int32_t n_kv_heads;
    // 8-bit caches: the pools hold bytes ([n_pages][Hkv][D/16][16][16] and [n_pages][Hkv][D][16]) and every
    // (page, head, slot) has an fp32 power-of-two scale for its key row and one for its value row
    // 4-bit caches: the pools hold codes, k_scale the scale bytes of both ([n_pages][Hkv][D]), see st_kv_cache
    float* k_scale;
    float* v_scale;
};

// the two 4-bit codes of byte `byte` (0 .. 3, a constant once loops are unrolled) as bf16 times the power of two in scale's exponent, all the conversion
// looks at there (all ones: NaN)
__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float scale, int byte) {
    switch (byte) {
        case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
        case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
        case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
        default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
}

__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
    bf16x2 r;
    r[0] = (__bf16)lo;
    r[1] = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, r);
}

st_status check_cache(const st_kv_cache& c, const char* who, const char* which, bool allow_fp8 = false, bool allow_fp4 = false);
CacheView cache_view(const st_kv_cache& c);
// One token per sequence into a (checked, bf16) cache at index len_after[b] - 1; the length becomes len_after[b].
st_status append_token_at(const st_kv_cache& c, const void* k_new, const void* v_new, const int32_t* len_after, int batch,
                          bool rotate, double theta_base, hipStream_t s);
// New tokens into a (checked) cache of any storage format: k_weight (null: not normalised), rope (null: not rotated), start_len (null:
// appended_len).
struct RopeTable;
st_status append_rows(const char* who, const st_kv_cache& c, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                      const int32_t* start_len, const int32_t* n_new, int max_new, int batch, const void* k_weight, double eps,
                      const RopeTable* rope, hipStream_t s);

}  // namespace st
