// Attention over binary16 rows for gfx950: one pass over the keys with the running maximum and sum of the softmax.
//
// A workgroup of NW wavefronts has 32 NW packed rows (attention.h) of one sequence and key head; keys and values go by tiles of 64 from global memory into
// LDS (global_load_lds, no registers), two tiles deep, and every wavefront reads them from there: attention_tile.h says how.
#include "attention_tile.h"

namespace ql {

template <int CHP, int NW, bool SHAPED>
__global__ __launch_bounds__(64 * NW, CHP <= 16 ? 2 : 1) void attend_tiles(AttnArgs a, TilePlan plan)
{
    attend_tile<CHP, NW, false, SHAPED>(a, plan);
}

__global__ __launch_bounds__(JOIN_THREADS) void join_tiles(AttnArgs a, TilePlan plan, int rows_per) { join_splits(a, plan, rows_per); }

namespace {
constexpr int CUS = 256;

// rows of a workgroup: as many as still give every CU one (long heads: the addresses of a tile that few wavefronts load take their registers)
int tile_rows(long long Tq, int B, int G, int Hkv, int D)
{
    for (int rows = 128; rows > (D > 128 ? 128 : D > 80 ? 64 : 32); rows /= 2)
        if ((Tq * G / rows + B) * Hkv >= CUS) return rows;
    return D > 128 ? 128 : D > 80 ? 64 : 32;
}

template <int CHP, int NW>
hipError_t launch_tiles(const AttnArgs &a, hipStream_t stream)
{
    using T = AttnTile<CHP, NW, false>;
    const TilePlan p = tile_plan(a.Tq, a.B, a.G, a.Hkv, T::ROWS, a.cu_q, a.mask, a.Tk / a.B, CUS, 2 * CUS);
    static const hipError_t opt_in[2] = {
        hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_tiles<CHP, NW, false>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES),
        hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_tiles<CHP, NW, true>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES)};
    const bool shaped = a.cap > 0.0f || a.slopes;
    if (opt_in[shaped] != hipSuccess) return opt_in[shaped];
    const long long wgs = (long long)p.tiles * a.Hkv * p.splits;
    const dim3 grid((unsigned)((wgs + 7) / 8 * 8));
    if (shaped) hipLaunchKernelGGL((attend_tiles<CHP, NW, true>), grid, dim3(T::NT), T::LDS_BYTES, stream, a, p);
    else hipLaunchKernelGGL((attend_tiles<CHP, NW, false>), grid, dim3(T::NT), T::LDS_BYTES, stream, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL(join_tiles, dim3((unsigned)(p.tiles * a.Hkv), join_blocks(T::ROWS, a.D)), dim3(JOIN_THREADS), 0, stream, a, p, T::ROWS);
    return hipGetLastError();
}

// rows: what tile_rows gave
hipError_t launch_by_head(const AttnArgs &a, int rows, hipStream_t stream)
{
    const int ch = a.D / 8;
    if (rows == 32) {
        if (ch <= 2) return launch_tiles<2, 1>(a, stream);
        if (ch <= 4) return launch_tiles<4, 1>(a, stream);
        if (ch <= 6) return launch_tiles<6, 1>(a, stream);
        if (ch <= 8) return launch_tiles<8, 1>(a, stream);
        if (ch == 9) return launch_tiles<9, 1>(a, stream);
        return launch_tiles<10, 1>(a, stream);
    }
    if (rows == 64) {
        if (ch <= 2) return launch_tiles<2, 2>(a, stream);
        if (ch <= 4) return launch_tiles<4, 2>(a, stream);
        if (ch <= 6) return launch_tiles<6, 2>(a, stream);
        if (ch <= 8) return launch_tiles<8, 2>(a, stream);
        if (ch == 9) return launch_tiles<9, 2>(a, stream);
        if (ch <= 10) return launch_tiles<10, 2>(a, stream);
        if (ch <= 12) return launch_tiles<12, 2>(a, stream);
        return launch_tiles<16, 2>(a, stream);
    }
    if (ch <= 2) return launch_tiles<2, 4>(a, stream);
    if (ch <= 4) return launch_tiles<4, 4>(a, stream);
    if (ch <= 6) return launch_tiles<6, 4>(a, stream);
    if (ch <= 8) return launch_tiles<8, 4>(a, stream);
    if (ch == 9) return launch_tiles<9, 4>(a, stream);
    if (ch <= 10) return launch_tiles<10, 4>(a, stream);
    if (ch <= 12) return launch_tiles<12, 4>(a, stream);
    if (ch <= 16) return launch_tiles<16, 4>(a, stream);
    if (ch <= 24) return launch_tiles<24, 4>(a, stream);
    return launch_tiles<32, 4>(a, stream);
}
}  // namespace

size_t tiles_partial_bytes(long long Tq, long long Tk, int B, int Hq, int Hkv, int D)
{
    const int rows = tile_rows(Tq, B, Hq / Hkv, Hkv, D);
    const TilePlan p = tile_plan(Tq, B, Hq / Hkv, Hkv, rows, true, 0, Tk / B, CUS, 2 * CUS);
    return p.splits == 1 ? 0 : (size_t)p.tiles * Hkv * p.splits * rows * (D + 2) * 4;
}

hipError_t launch_attention_f16(const AttnArgs &a, hipStream_t stream)
{
    const int rows = tile_rows(a.Tq, a.B, a.G, a.Hkv, a.D);
    return launch_by_head(a, rows, stream);
}

}  // namespace ql
