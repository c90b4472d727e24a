// Dynamic quantization to e4m3 with a scale for every row and 128 channels (gfx950): of binary16 rows, of the gated product silu(g) * u that
// rows [g | u] stand for, and of fp32 rows (the experts' gated products).
//
// scale = amax / 448 of a block's values v, code = e4m3 nearest to 448 v / amax (f8.h).  Bound by memory: 3 bytes a value (5 gated) and about 12 vector instructions (31
// gated, whose busy cycles the vector units fill, too).  16 lanes own a block, 8 values each: a 16-byte load, the maximum over 16 lanes by rotations inside the row of lanes,
// an 8-byte store, nothing is read twice.  A copy moves 5.0 TB/s; 16384 x 4608 takes 38 us (6.0 TB/s, part of it from the caches), gated 77 us (4.9 TB/s), from memory 82; 16 x 4096 2.7 us.
#include "daq_f8.h"

namespace ql {

template <bool GLU, bool WIDE>
__global__ __launch_bounds__(256) void daq_f8(F8DaqArgs a)
{
    daq_f8_blocks<GLU, WIDE>(a, (long long)blockIdx.x * 16 + (threadIdx.x >> 4), (long long)gridDim.x * 16);
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
