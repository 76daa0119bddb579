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

// distance of a tile's piece of 16 features from its beginning, in the descriptors' unit
__device__ __forceinline__ constexpr uint32_t piece(int k) { return ((k / 4) * (128 * 128) + (k % 4) * 32) / 16; }

// ---- The items of a block (a tile, or a part of one) are found by a warp of their own and handed to the others through shared memory, a few
// ahead: where a segment lies comes from global memory, and the kernels' shared memory leaves no first-level cache, so every warp that
// looked for itself (or kept the walk's state in spilled registers) stood still for thousands of cycles between items.
constexpr int ITEMS = 4;
struct Item {
    int q0, nq, k0, nk, length, s, h, t, steps, i0, i1;     // as in Walker; steps 0: there are no more
    __device__ __forceinline__ Segment segment() const { return {q0, nq, k0, nk, length}; }
};
struct ItemRing {
    unsigned long long full[ITEMS], empty[ITEMS];
    Item item[ITEMS], none;         // none: in place of the items that were not handed out
    uint32_t given_up;              // the first of these
    float factor[ITEMS];            // what the kernel says of an item's segment (apart from the items, whose twelfth word would change how all warps load them)
};
__device__ __forceinline__ void items_init(ItemRing& r, int consumer_warps) {
    r.none.steps = 0;
    r.given_up = ~0u;
    for (int i = 0; i < ITEMS; ++i) { mbar_init(smem_u32(&r.full[i]), 1); mbar_init(smem_u32(&r.empty[i]), consumer_warps); }
}
struct NoFactor {
    __device__ __forceinline__ float operator()(int) const { return 1.f; }
};
// Waits at most `limit` cycles for the return of an item; then there are no more, and every warp learns from which one on.
template <typename W, typename F = NoFactor>
__device__ __forceinline__ void items_hand_out(ItemRing& r, const AttnParams& p, W& it, bool more, long long limit = A_MINUTE, F factor = F()) {
    for (uint32_t n = 0;; ++n) {
        if (n >= (uint32_t)ITEMS && !mbar_wait_for(smem_u32(&r.empty[n % ITEMS]), (n / ITEMS + 1) & 1, limit)) {
            __threadfence_block();
            *(volatile uint32_t*)&r.given_up = n;
            return;
        }
        r.item[n % ITEMS] = {it.g.q0, it.g.nq, it.g.k0, it.g.nk, it.g.length, it.s, it.h, it.t, more ? it.steps : 0, it.i0, it.i1};
        if (more) r.factor[n % ITEMS] = factor(it.s);
        mbar_arrive(smem_u32(&r.full[n % ITEMS]));
        if (!more) return;
        more = it.next(p);
    }
}
// What a block leaves for the kernel that joins: the tile that ends in its first item and began in an earlier block's (parts 0: none).
struct Joint {
    Item item;
    int first, parts;           // the block in which the tile begins; how many share it
};
template <typename C>
__device__ __forceinline__ Joint joint_of(const AttnParams& p, const Walker<C>& it, bool any, int block) {
    Joint j;
    j.item = {it.g.q0, it.g.nq, it.g.k0, it.g.nk, it.g.length, it.s, it.h, it.t, it.steps, it.i0, it.i1};
    const bool ends = any && it.i0 > 0 && it.i1 == it.steps;
    j.first = ends ? it.first_block(p, block) : 0;
    j.parts = ends ? block - j.first + 1 : 0;
    return j;
}
// The n-th item, for a whole warp, and its return.  Neither looks at the abort word: every warp goes through all items.  A warp does not
// give up by itself: warps that meet at a barrier have to leave at the same item.  The warp that hands out does so for all of them after a
// minute at most, so this wait ends as well (a bound of its own, four minutes, lies behind that): items in front of given_up are there.
__device__ __forceinline__ const Item& item_take(ItemRing& r, uint32_t n) {
    const long long t0 = clock64();
    uint32_t end = ~0u;
    while (!mbar_try(smem_u32(&r.full[n % ITEMS]), (n / ITEMS) & 1)) {
        end = *(volatile uint32_t*)&r.given_up;
        if (end == ~0u && clock64() - t0 > 4 * A_MINUTE) end = 0;
        if (end != ~0u) {
            __threadfence_block();
            break;
        }
    }
    const bool came = __all_sync(~0u, n < end);
    return came ? r.item[n % ITEMS] : r.none;
}
__device__ __forceinline__ void item_return(ItemRing& r, uint32_t n) {
    __syncwarp();
    if (threadIdx.x % 32 == 0) mbar_arrive(smem_u32(&r.empty[n % ITEMS]));
}

// Tensor maps of the arrays: q and grad_out as [rows][heads][D], boxes of 32 packed rows of a kv head (32 / group rows of its group
// heads: one box where group divides 32); key and value as [heads][rows][D] or [pages][heads][slots][D], boxes of kv_box rows of a head.
struct TileMaps { CUtensorMap q, go, k, v; };

// 32 rows of a tile by one warp, and its 32 arrivals on the barrier.  Rows that all exist come in boxes (lane l holds the coordinates of
// the box that begins at its row), issued by one lane each; rows of which some are masked, missing or behind the end come one by one.
// (With copies of 16 bytes alone, the addresses cost a producer warp about 2000 instructions a step and bounded the kernels: chunk of
// 2048 on 16384 508 us with the softmax left out.)
template <int DP>
__device__ __forceinline__ void fetch_rows(uint32_t tile, int first_row, uint32_t bar, int box, const CUtensorMap* map, int c1, int c2, int c3,
                                           const void* base, long long off, int D, const void* any) {
    if (box && __all_sync(~0u, off >= 0)) {
        const int lane = threadIdx.x % 32;
        if (lane == 0) { mbar_arrive(bar, 31); mbar_arrive_expect(bar, 32 * DP * 2); }
        __syncwarp();
        if (lane % box == 0)
#pragma unroll
            for (int f = 0; f < DP / 64; ++f) box_copy(tile + f * (128 * 128) + (first_row + lane) * 128, map, bar, 64 * f, c1, c2, c3);
    } else {
        copy_rows<DP, 128, 32>(tile, first_row, base, off, D, any);
        cp_async_arrive(bar);
    }
}
template <int DP>
__device__ __forceinline__ void fetch_keys(uint32_t tile, int first_row, uint32_t bar, const AttnParams& p, const TileMaps& m, bool values, Place a, int h, const void* any) {
    fetch_rows<DP>(tile, first_row, bar, p.kv_box, values ? &m.v : &m.k, p.table ? a.slot : a.at, h, p.table ? a.at : 0, values ? p.v : p.k,
                   values ? value_offset(p, a, h) : key_offset(p, a, h), p.D, any);
}
// lane l's packed row is first + l of kv head h; `on`: it exists and is wanted
template <int DP>
__device__ __forceinline__ void fetch_packed(uint32_t tile, int first_row, uint32_t bar, const AttnParams& p, const Segment& g, const TileMaps& m, bool grads, int h, int r, bool on, const void* any) {
    const PackedRow pr = packed_row(p, g, h, on ? r : 0);
    fetch_rows<DP>(tile, first_row, bar, p.q_box, grads ? &m.go : &m.q, h * p.group, pr.row, 0, grads ? p.go : p.q,
                   !on ? -1 : grads ? pr.row * p.go_row + pr.head * p.go_head : pr.row * p.q_row + pr.head * p.q_head, p.D, any);
}

// A warp's lanes each hold C pieces of 16 bytes of a row of their own, to be written at `to` (those of them below `wanted`; `on`: the row
// exists).  C lanes exchange pieces first, so that they write one row's together: a store instruction then touches 32 / C lines and whole
// sectors, not 32 lines and half sectors (which took 2000 cycles for every 16 features of a tile, a third of an item of six steps).
template <int C>
__device__ __forceinline__ void store_rows(uint4 (&v)[C], void* to, bool on, int wanted) {
    const int lane = threadIdx.x % 32, q = lane % C;
#pragma unroll
    for (int s = 1; s < C; s *= 2)
#pragma unroll
        for (int a = 0; a < C; ++a) {
            if (a & s) continue;
            const bool up = q & s;
            uint4 t = up ? v[a] : v[a | s];
            t.x = __shfl_xor_sync(~0u, t.x, s);
            t.y = __shfl_xor_sync(~0u, t.y, s);
            t.z = __shfl_xor_sync(~0u, t.z, s);
            t.w = __shfl_xor_sync(~0u, t.w, s);
            if (up) v[a] = t; else v[a | s] = t;
        }
    const unsigned rows = __ballot_sync(~0u, on);
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int from = lane - q + j;
        const unsigned long long base = __shfl_sync(~0u, (unsigned long long)to, from);
        if ((rows >> from & 1) && q < wanted) *reinterpret_cast<uint4*>(base + 16 * q) = v[j];
    }
}

// 32 bytes, on a boundary of 32, by one lane
__device__ __forceinline__ void store_sector(void* to, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// Two pieces of each lane's row: a store of 32 bytes where the rows' pieces lie on whole sectors, which needs no exchange.
__device__ __forceinline__ void store_pieces(uint4 (&v)[2], void* to, bool on, int wanted, bool whole_sectors) {
    if (whole_sectors) {
        const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
        if (on && wanted > 0) store_sector(to, w);
    } else store_rows<2>(v, to, on, wanted);
}

// host: the maps, and the boxes that they allow (attention.cu)
void make_tile_maps(AttnParams* p, bool bf16, TileMaps* m);
bool make_row_map(const AttnParams& p, bool bf16, int packed, CUtensorMap* m);

// blocks of the persistent kernels: one on every SM (their shared memory admits one), 0 if the device does not answer
static inline int attention_grid() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms < MAX_SMS ? sms : MAX_SMS;
}

}  // namespace tiga
