// Attention over dense and paged relations: what the kernels and the host share.
#pragma once
#include <cuda_bf16.h>
#include <math.h>
#include "common.cuh"

namespace tiga {

constexpr float LOG2E_F = 1.4426950408889634f, LN2_F = 0.6931471805599453f;

struct AttnParams {
    const void *q, *k, *v, *o, *go;
    void *out, *gq, *gk, *gv;
    float* lse;
    const float* lse_in;
    long long q_row, q_head, k_row, k_head, v_row, v_head, go_row, go_head;
    const int32_t *q_start, *kv_start, *kv_len, *table;      // table: NULL for the dense relation
    const uint8_t* mask;
    int n_seg, n_q, n_kv, heads, kv_heads, group, D, causal;
    long long n_pages, page_size, table_stride, max_pages, page_stride, slot_stride;
    float scale;
};

// A segment's rows [q0, q0 + nq) and its keys [k0, k0 + nk) (paged: k0 = 0), bounds clamped to the arrays.
struct Segment { int q0, nq, k0, nk; };

__device__ __forceinline__ int clamp_to(int v, int hi) { return min(max(v, 0), hi); }

__device__ __forceinline__ Segment segment_of(const AttnParams& p, int s) {
    Segment g;
    g.q0 = clamp_to(p.q_start[s], p.n_q);
    g.nq = max(clamp_to(p.q_start[s + 1], p.n_q) - g.q0, 0);
    if (p.table) {
        g.k0 = 0;
        g.nk = (int)min((long long)max(p.kv_len[s], 0), p.max_pages * p.page_size);
    } else {
        g.k0 = clamp_to(p.kv_start[s], p.n_kv);
        g.nk = max(clamp_to(p.kv_start[s + 1], p.n_kv) - g.k0, 0);
    }
    return g;
}

// keys that row t of the segment's nq rows reads: [0, this)
__device__ __forceinline__ int keys_of_row(const AttnParams& p, const Segment& g, int t) {
    return p.causal ? min(max(g.nk - g.nq + t + 1, 0), g.nk) : g.nk;
}

// Where key j of segment s (0 <= j < g.nk) lies, or -1 where it is masked or has no page.  Paged: the offset of its slot in either
// array, in elements (row_scale 1).  Dense: its row (row_scale: the row stride of the array that is read).
__device__ __forceinline__ long long key_place(const AttnParams& p, const Segment& g, int s, int j) {
    if (p.table) {
        const int page = j / (int)p.page_size;
        const int id = p.table[(long long)s * p.table_stride + page];
        if (id < 0 || id >= p.n_pages) return -1;
        return (long long)id * p.page_stride + (long long)(j - page * (int)p.page_size) * p.slot_stride;
    }
    if (p.mask && !p.mask[g.k0 + j]) return -1;
    return g.k0 + j;
}

// ---- How the work is cut.  A segment's heads share keys, so the rows of a group's heads are packed: packed row r of a kv head is row
// r / group, head kv_head * group + r % group.  A tile of stationary rows (packed rows, or keys for their gradients) meets the other
// side in steps; a unit is one step of one tile of one kv head.  All units of a call stand in one line (segment, kv head, tile,
// step), and the blocks take equal pieces of it: a piece that begins or ends inside a tile leaves a partial state in the
// workspace, and a last kernel joins those in order.  So short and long, few and many rows are balanced by one rule.
struct Geometry { int tile, step, keys_stationary; };

__device__ __forceinline__ int stationary_rows(const AttnParams& p, const Segment& g, const Geometry geo) {
    return geo.keys_stationary ? g.nk : g.nq * p.group;
}
__device__ __forceinline__ int tiles_of(const AttnParams& p, const Segment& g, const Geometry geo) {
    return (int)(((long long)stationary_rows(p, g, geo) + geo.tile - 1) / geo.tile);
}
// steps of tile t; one (in which nothing is read) where there is nothing on the other side, so that empty rows are written
__device__ __forceinline__ int steps_of(const AttnParams& p, const Segment& g, const Geometry geo, int t) {
    long long n;
    if (geo.keys_stationary) n = (long long)g.nq * p.group;
    else if (!p.causal) n = g.nk;
    else {
        const long long last = min(((long long)t + 1) * geo.tile, (long long)g.nq * p.group) - 1;
        n = keys_of_row(p, g, (int)(last / p.group));
    }
    return (int)max((n + geo.step - 1) / geo.step, 1LL);
}
__device__ __forceinline__ long long units_of_head(const AttnParams& p, const Segment& g, const Geometry geo) {
    const int tiles = tiles_of(p, g, geo);
    if (!p.causal || geo.keys_stationary) return (long long)tiles * (tiles ? steps_of(p, g, geo, 0) : 0);
    long long n = 0;
    for (int t = 0; t < tiles; ++t) n += steps_of(p, g, geo, t);
    return n;
}

// Blocks that take part: `least` units each at least, so that tiny work is not spread thin.
__device__ __forceinline__ long long blocks_for(long long units, int grid, int least) {
    return min((long long)grid, max((units + least - 1) / least, 1LL));
}

// A block's way through its piece of the line: one tile, or a part of one, after the other.
struct Walker {
    Segment g;
    int s, h, t;                // segment, kv head, tile
    int steps, i0, i1;          // steps of the tile, and which of them are this block's
    long long left;             // units behind this item

    __device__ __forceinline__ void open(const AttnParams& p, const Geometry geo) {
        steps = steps_of(p, g, geo, t);
        i1 = (int)min((long long)steps, i0 + left);
        left -= i1 - i0;
    }
    // false: the piece is empty
    __device__ __forceinline__ bool begin(const AttnParams& p, const Geometry geo, const long long* unit_start, long long unit, long long end) {
        left = end - unit;
        if (left <= 0) return false;
        int lo = 0, hi = p.n_seg;               // the last segment that begins at or before this unit
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (unit_start[mid] <= unit) lo = mid; else hi = mid;
        }
        s = lo;
        g = segment_of(p, s);
        long long off = unit - unit_start[s];
        const long long per_head = (unit_start[s + 1] - unit_start[s]) / p.kv_heads;
        h = (int)(off / per_head);
        off -= h * per_head;
        if (!p.causal || geo.keys_stationary) {
            const int n = steps_of(p, g, geo, 0);
            t = (int)(off / n);
            i0 = (int)(off - (long long)t * n);
        } else {
            t = 0;
            for (int n; off >= (n = steps_of(p, g, geo, t)); ++t) off -= n;
            i0 = (int)off;
        }
        open(p, geo);
        return true;
    }
    __device__ __forceinline__ bool next(const AttnParams& p, const Geometry geo) {
        if (left <= 0) return false;
        i0 = 0;
        if (++t >= tiles_of(p, g, geo)) {
            t = 0;
            if (++h >= p.kv_heads) {
                h = 0;
                do { g = segment_of(p, ++s); } while (tiles_of(p, g, geo) == 0);
            }
        }
        open(p, geo);
        return true;
    }
};

// unit_start[s]: units in front of segment s.  By one block.
constexpr int PLAN_THREADS = 1024;
static __device__ void plan_units(const AttnParams& p, const Geometry geo, long long* unit_start) {
    __shared__ long long warp_total[PLAN_THREADS / 32];
    long long before = 0;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int s0 = 0; s0 < p.n_seg; s0 += PLAN_THREADS) {
        const int s = s0 + threadIdx.x;
        long long n = 0;
        if (s < p.n_seg) n = units_of_head(p, segment_of(p, s), geo) * p.kv_heads;
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(~0u, n, o);
            if (lane >= o) n += v;
        }
        if (lane == 31) warp_total[warp] = n;
        __syncthreads();
        long long sum = before;
        for (int w = 0; w < PLAN_THREADS / 32; ++w) {
            if (w < warp) sum += warp_total[w];
            before += warp_total[w];
        }
        if (s < p.n_seg) unit_start[s + 1] = sum + n;
        __syncthreads();
    }
    if (threadIdx.x == 0) unit_start[0] = 0;
}

constexpr int MAX_SMS = 160;            // blocks that workspaces provide for

size_t attention_forward_bytes(const AttnParams& p);
size_t attention_backward_bytes(const AttnParams& p);
tiga_status attention_backward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s);
tiga_status attention_forward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s);

// host checks of the descriptors (attention.cu)
tiga_status attention_heads_check(const tiga_heads* h);
tiga_status attention_pages_check(const tiga_pages* c);
bool attention_bad_stride(const tiga_stride& s);

template <typename T> struct Half;
template <> struct Half<__half> {
    static __device__ __forceinline__ float to(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from(float v) { return __float2half_rn(v); }
};
template <> struct Half<__nv_bfloat16> {
    static __device__ __forceinline__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Half<float> {
    static __device__ __forceinline__ float to(float v) { return v; }
    static __device__ __forceinline__ float from(float v) { return v; }
};

}  // namespace tiga
