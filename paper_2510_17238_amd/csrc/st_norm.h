// Rotation by a caller's st_rope_spec, and what the kernels that normalise rows share (internal).
#pragma once
#include <type_traits>

#include "st_internal.h"

namespace st {

// A spec turned into what a kernel needs: the angle per position of every rotated pair, in 64 bits.
struct RopeTable {
    double f[64];
    int rot;            // leading dims that are rotated (a multiple of 16)
    int interleaved;    // pairs (2 i, 2 i + 1) instead of (i, i + rot / 2)
    double a;           // factor on the rotated dims
};
// Checks the spec and forms the table (ST_OK), or says what is wrong with it.
st_status make_rope_table(const char* who, const st_rope_spec* spec, int head_dim, RopeTable* table);

// A lane's place in a rotation, c the lane's place in its row: the lane that holds the partners of its dims, the first of its pairs, whether any of its
// dims are rotated, whether they are the second halves of their pairs.
struct RowTurn {
    int partner, at;
    bool turned, high;
    __device__ __forceinline__ RowTurn(const RopeTable& rope, int c) {
        const int half = rope.rot / 2;
        high = 8 * c >= half;
        turned = 8 * c < rope.rot;
        partner = (int(threadIdx.x) & 63) + (turned ? (high ? -half / 8 : half / 8) : 0);
        at = rope.interleaved ? 4 * c : high ? 8 * c - half : 8 * c;
    }
};

// A row (one token of one head) lies in D / 8 neighbouring lanes, eight dims each.  Sum over those lanes, by data-parallel
// moves: neighbours, pairs, halves of eight mirrored, of sixteen mirrored.
template <int LANES, typename F>
__device__ __forceinline__ F row_sum(F x) {
    static_assert(LANES == 8 || LANES == 16, "head_dim 64 or 128");
    auto dpp = [](F v, auto ctrl) {
        constexpr int C = decltype(ctrl)::value;
        if constexpr (sizeof(F) == 4) {
            return __builtin_bit_cast(F, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), C, 0xf, 0xf, true));
        } else {
            u32x2 u = __builtin_bit_cast(u32x2, v);
            u[0] = uint32_t(__builtin_amdgcn_update_dpp(0, int(u[0]), C, 0xf, 0xf, true));
            u[1] = uint32_t(__builtin_amdgcn_update_dpp(0, int(u[1]), C, 0xf, 0xf, true));
            return __builtin_bit_cast(F, u);
        }
    };
    x += dpp(x, std::integral_constant<int, 0xb1>{});       // quad_perm 1,0,3,2
    x += dpp(x, std::integral_constant<int, 0x4e>{});       // quad_perm 2,3,0,1
    x += dpp(x, std::integral_constant<int, 0x141>{});      // mirrored within eight
    if constexpr (LANES == 16) x += dpp(x, std::integral_constant<int, 0x140>{});       // mirrored within sixteen
    return x;
}

}  // namespace st
