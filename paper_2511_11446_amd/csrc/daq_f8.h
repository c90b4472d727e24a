// A wavefront's part of the dynamic quantization to e4m3: of the kernel of that (daq_f8.hip) and of one that has workgroups to spare (route.hip).
#pragma once
#include "daq_device.h"
#include "f8.h"

namespace ql {

// Blocks first, first + step, ... of 128 channels (block KB m + b of row m), each by 16 neighbouring lanes
template <bool GLU, bool WIDE>
__device__ __forceinline__ void daq_f8_blocks(const F8DaqArgs &a, long long first, long long step)
{
    const int sub = threadIdx.x & 15;
    const long long rows = a.rows ? min(*a.rows, a.M) : a.M;
    for (long long g = first; g < rows * a.KB; g += step) {
        const long long m = g / a.KB;
        const int b = (int)(g - m * a.KB), k = b * F8_BLOCK + sub * 8;
        float v[8];
        if (k < a.K) {
            if constexpr (WIDE) {
                const float *x = static_cast<const float *>(a.x) + m * a.K + k;
                const float4 lo = *reinterpret_cast<const float4 *>(x), hi = *reinterpret_cast<const float4 *>(x + 4);
                v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
            } else {
                const _Float16 *x = static_cast<const _Float16 *>(a.x) + m * a.K * (GLU ? 2 : 1) + k;
                typedef _Float16 h8 __attribute__((ext_vector_type(8)));
                const h8 p = *reinterpret_cast<const h8 *>(x);
                h8 u = p;
                if constexpr (GLU) u = *reinterpret_cast<const h8 *>(x + a.K);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = GLU ? silu_dev((float)p[i]) * (float)u[i] : (float)p[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        }
        float m8 = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m8 = fmaxf(m8, fabsf(v[i]));
        const float amax = max16(m8);
        const F8Scale s(amax);
        if (k < a.K) {
            uint2 out;
            out.x = f8_pack4(s.code(v[0]), s.code(v[1]), s.code(v[2]), s.code(v[3]));
            out.y = f8_pack4(s.code(v[4]), s.code(v[5]), s.code(v[6]), s.code(v[7]));
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.q) + m * a.K + k) = out;
        }
        if (sub == 0) a.scales[m * a.KB + b] = F8Scale::scale(amax);
    }
}

}  // namespace ql
