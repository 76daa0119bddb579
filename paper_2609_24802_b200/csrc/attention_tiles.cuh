// What the forward and the backward kernels do alike: rows of a packed tile, copies of rows into swizzled tiles, the grid.
#pragma once
#include "attention_shared.cuh"
#include "tcgen.cuh"

namespace tiga {

// packed row r of kv head h: offsets of its row in arrays with strides
struct PackedRow { int row, head; };
__device__ __forceinline__ PackedRow packed_row(const AttnParams& p, const Segment& g, int h, int r) {
    const int t = r / p.group;
    return {g.q0 + t, h * p.group + (r - t * p.group)};
}

// ROWS rows of a tile by one warp: lane l (< ROWS) holds row l's element offset (or -1: zeros; `any` is an
// address that may be read).  The tile consists of blocks of 64 features, rows
// of 128 bytes swizzled in groups of eight.
template <int DP, int TILE_ROWS, int ROWS>
__device__ __forceinline__ void copy_rows(uint32_t tile, int first_row, const void* base, long long off, int D, const void* any) {
    constexpr int CH = DP / 8;
    const int lane = threadIdx.x % 32, c = lane % CH;
    const bool in_width = c * 8 < D;
#pragma unroll
    for (int k = 0; k < ROWS * CH / 32; ++k) {
        const int r = k * (32 / CH) + lane / CH;
        const long long o = __shfl_sync(~0u, off, r);
        const int row = first_row + r;
        const bool on = o >= 0 && in_width;
        cp_async16(tile + (c / 8) * (TILE_ROWS * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4),
                   on ? (const char*)base + (o + c * 8) * 2 : (const char*)any, on);
    }
}

// blocks of the persistent kernels: one on every SM (their shared memory admits one), 0 if the device does not answer
static inline int attention_grid() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms < MAX_SMS ? sms : MAX_SMS;
}

}  // namespace tiga
