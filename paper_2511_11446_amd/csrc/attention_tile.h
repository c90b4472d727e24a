// The tile of attention: a wavefront's 32 packed rows against 64 keys at a time (attention.hip).  Not part of the public ABI.
//
// Scores come as S^T = K Q^T (mfma 32x32x16): a lane has ONE row (lane & 31) and 16 of 32 keys, so the running maximum and sum of a row
// are the lane's own up to one exchange with lane ^ 32, masks and biases know the row without an index, and the weights are in the
// place where O^T = V^T P^T wants its right operand: keys 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4 of a lane are slots j of step s on
// both sides, whatever their order.  V^T comes out of the row-major tile by the transposing LDS read (4 keys of 16 channels).
#pragma once
#include "attention.h"

namespace ql {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void attn_lds;
typedef const __attribute__((address_space(1))) void attn_global;
typedef __attribute__((address_space(3))) s16x4 attn_lds_s4;

constexpr int ATT_KEYS = 64;   // keys of a tile
constexpr float LOG2E = 1.4426950408889634f;

// CHP: 16-byte pieces of a tile row (D / 8 rounded up to a multiple of 2).  A row is kept without padding (a wavefront's DMA fills 1024
// neighbouring bytes); the piece c of row r sits at slot c ^ f(r), so that 8 rows read at one piece index (keys) and 4 rows read at 4
// neighbouring ones (values) spread over all banks.
template <int CHP> __device__ __forceinline__ constexpr int key_swizzle(int r)
{
    return CHP % 16 == 0 ? (r & 7) : CHP % 16 == 8 ? (r >> 1 & 7) : CHP % 4 == 0 ? (r >> 2 & 3) : 0;
}
template <int CHP> __device__ __forceinline__ constexpr int value_swizzle(int r)
{
    return CHP % 16 == 0 ? (r & 3) << 2 : CHP % 16 == 8 ? (r >> 1 & 1) << 2 : 0;
}

// a lane's value and that of lane ^ 32, which has the same row (the two results are taken out as whole words first: a bit cast of a vector
// element reads element 0)
struct Halves {
    float a, b;
};
__device__ __forceinline__ Halves both_halves(float x)
{
    const unsigned w = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const unsigned a = r[0], b = r[1];
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// cap * tanh(x / cap) from x / cap * 2 log2(e) (t): 1 - 2 / (1 + e^2x), absolute error about 1e-7 of the cap
__device__ __forceinline__ float capped(float t, float cap) { return cap - 2.0f * cap * __builtin_amdgcn_rcpf(1.0f + exp2_fast(t)); }

}  // namespace ql
