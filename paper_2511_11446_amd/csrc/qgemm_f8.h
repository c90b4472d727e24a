// What the kernels of the products in 8-bit floating point share.  Not part of the public ABI.
#pragma once
#include "f8.h"
#include "qgemm_common.h"

namespace ql {

// a layer's epilogue: u, the fp32 value -> h = fp16(act(u)), then fma(gate, h, residual)
__device__ __forceinline__ void finish4(const F8Gemm &a, int m, int n, float (&u)[4])
{
    const _Float16 *bias = static_cast<const _Float16 *>(a.bias), *res = static_cast<const _Float16 *>(a.residual), *gate = static_cast<const _Float16 *>(a.gate);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int c = min(n + r, a.N - 1);
        if (bias) u[r] += (float)bias[c];
        if (a.act == 1) u[r] = gelu_tanh_dev(u[r]);
        if (res || gate) {
            asm volatile("" : "+v"(u[r]));
            const float h = (float)(_Float16)u[r];
            u[r] = __builtin_fmaf(gate ? (float)gate[(long long)(m / a.gate_rows) * a.N + c] : 1.0f, h, res ? (float)res[(long long)m * a.N + c] : 0.0f);
        }
        asm volatile("" : "+v"(u[r]));   // the fp32 value is rounded to fp16 in the store and nowhere earlier
    }
}

}  // namespace ql
