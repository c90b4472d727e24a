// Dynamic quantization to e4m3 with a scale for every row and 128 channels (gfx950): of binary16 rows, of the gated product silu(g) * u that
// rows [g | u] stand for, and of fp32 rows (the experts' gated products).
//
// scale = amax / 448 of a block's values v, code = e4m3 nearest to 448 v / amax (f8.h).  Bound by memory: 3 bytes a value (5 gated) and about 12 vector instructions (31
// gated, whose busy cycles the vector units fill, too).  16 lanes own a block, 8 values each: a 16-byte load, the maximum over 16 lanes by rotations inside the row of lanes,
// an 8-byte store, nothing is read twice.  A copy moves 5.0 TB/s; 16384 x 4608 takes 38 us (6.0 TB/s, part of it from the caches), gated 77 us (4.9 TB/s); 16 x 4096 2.8 us.
#include "daq_device.h"
#include "f8.h"

namespace ql {

template <bool GLU, bool WIDE>
__global__ __launch_bounds__(256) void daq_f8(F8DaqArgs a)
{
    const int sub = threadIdx.x & 15;
    const long long group = (long long)blockIdx.x * 16 + (threadIdx.x >> 4), step = (long long)gridDim.x * 16;
    const long long rows = a.rows ? min(*a.rows, a.M) : a.M;
    for (long long g = group; g < rows * a.KB; g += step) {
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

hipError_t launch_daq_f8(const F8DaqArgs &a, hipStream_t stream)
{
    const long long blocks = ((long long)a.M * a.KB + 15) / 16;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
    if (a.wide) hipLaunchKernelGGL((daq_f8<false, true>), grid, dim3(256), 0, stream, a);
    else if (a.glu) hipLaunchKernelGGL((daq_f8<true, false>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((daq_f8<false, false>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ql
