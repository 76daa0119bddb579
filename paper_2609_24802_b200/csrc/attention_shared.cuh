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
    int kv_box, q_box;              // rows that a box of the tensor maps brings (0: rows are copied one by one)
};

// A segment's rows [q0, q0 + nq) and its keys [k0, k0 + nk) (paged: k0 = 0), bounds clamped to the arrays.  length: its tokens, of which a
// cache may hold fewer (the rows' positions count from its end, not from that of the table).
struct Segment { int q0, nq, k0, nk, length; };

// Rows and positions end here, so that a tile's last row number fits 32 bits.
constexpr long long MOST_ROWS = 0x7fff0000LL;

__device__ __forceinline__ int clamp_to(int v, int hi) { return min(max(v, 0), hi); }

// (the bounds of rows and of dense keys: p.q_start and p.kv_start, or a copy of them)
__device__ __forceinline__ Segment segment_of(const AttnParams& p, int s, const int32_t* q_start, const int32_t* kv_start) {
    Segment g;
    g.q0 = clamp_to(q_start[s], p.n_q);
    g.nq = max(clamp_to(q_start[s + 1], p.n_q) - g.q0, 0);
    if (p.table) {
        g.k0 = 0;
        g.length = max(p.kv_len[s], 0);
        g.nk = (int)min(min((long long)g.length, p.max_pages * p.page_size), MOST_ROWS);
    } else {
        g.k0 = clamp_to(kv_start[s], p.n_kv);
        g.length = g.nk = max(clamp_to(kv_start[s + 1], p.n_kv) - g.k0, 0);
    }
    return g;
}
__device__ __forceinline__ Segment segment_of(const AttnParams& p, int s) { return segment_of(p, s, p.q_start, p.kv_start); }

// keys that row t of the segment's nq rows reads: [0, this)
__device__ __forceinline__ int keys_of_row(const AttnParams& p, const Segment& g, int t) {
    return p.causal ? min(max(g.length - g.nq + t + 1, 0), g.nk) : g.nk;
}

// Where key j of segment s (0 <= j < g.nk) lies: paged, its page and slot; dense, its row and 0.  at < 0: it is masked, or has no page.
struct Place { int at, slot; };
__device__ __forceinline__ Place key_place(const AttnParams& p, const Segment& g, int s, int j) {
    if (p.table) {
        const int page = j / (int)p.page_size;
        const int id = p.table[(long long)s * p.table_stride + page];
        return {id >= p.n_pages ? -1 : id, j - page * (int)p.page_size};
    }
    if (p.mask && !p.mask[g.k0 + j]) return {-1, 0};
    return {g.k0 + j, 0};
}
__device__ __forceinline__ long long key_offset(const AttnParams& p, Place a, int h) {
    return a.at < 0 ? -1 : p.table ? a.at * p.page_stride + a.slot * p.slot_stride + h * p.k_head : a.at * p.k_row + h * p.k_head;
}
__device__ __forceinline__ long long value_offset(const AttnParams& p, Place a, int h) {
    return a.at < 0 ? -1 : p.table ? a.at * p.page_stride + a.slot * p.slot_stride + h * p.v_head : a.at * p.v_row + h * p.v_head;
}

// Whether the rows of a dense segment read one key: its weight is 1 whatever the score, so scores have no gradient.  (Masks of up to
// 32 keys are counted; where a longer one leaves a single key the gradient is what is left of dP - delta, a few 2^-23 of either.)
__device__ __forceinline__ bool reads_one_key(const AttnParams& p, const Segment& g) {
    if (!p.mask || g.nk > 32) return g.nk == 1;
    int n = 0;
    for (int j = 0; j < g.nk; ++j) n += p.mask[g.k0 + j] != 0;
    return n == 1;
}

// the segment that holds row i (the last one that starts at or before it), or -1
__device__ __forceinline__ int segment_of_row(const int32_t* start, int n_seg, int n_rows, int i) {
    int lo = 0, hi = n_seg;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= i) lo = mid + 1; else hi = mid;
    }
    if (lo == 0 || i >= clamp_to(start[lo], n_rows)) return -1;
    return lo - 1;
}

// The last of n ascending places that is at most `v`, which start[0] is: by a warp with all its lanes, 32 places a round.
template <typename V>
__device__ __forceinline__ int last_place(const V* start, int n, V v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int gap = (hi - lo + 31) / 32, at = lo + (int)(threadIdx.x % 32) * gap;
        const unsigned before = __ballot_sync(~0u, at < hi && start[at] <= v) | 1u;
        lo += (31 - __clz(before)) * gap;
        hi = min(hi, lo + gap);
    }
    return lo;
}

// The segment of rows that come one behind the other.  A segment's end is kept; behind it the next one is sought in growing strides (there
// may be many without rows in between).
struct Along {
    int s, end;
    __device__ __forceinline__ void open(const int32_t* start, int n_seg, int row) {            // by a whole warp
        s = last_place(start, n_seg, row);
        end = s + 1 < n_seg ? start[s + 1] : INT32_MAX;
    }
    __device__ __forceinline__ bool go_on(const int32_t* start, int n_seg, int row) {           // true: to another segment
        if (row < end) return false;
        int lo = s + 1, hi = lo + 1;                // start[lo] <= row
        while (hi < n_seg && start[hi] <= row) { const int step = 2 * (hi - lo); lo = hi; hi = lo + step; }
        hi = min(hi, n_seg);
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= row) lo = mid; else hi = mid;
        }
        s = lo;
        end = s + 1 < n_seg ? start[s + 1] : INT32_MAX;
        return true;
    }
};

// ---- How the work is cut.  A segment's heads share keys, so the rows of a group's heads are packed: packed row r of a kv head is row
// r / group, head kv_head * group + r % group.  A tile of stationary rows (packed rows, or keys for their gradients) meets the other
// side in steps; a unit is one step of one tile of one kv head.  All units of a call stand in one line (segment, kv head, tile,
// step), and the blocks take equal pieces of it: a piece that begins or ends inside a tile leaves a partial state in the
// workspace, and a last kernel joins those in order.  So short and long, few and many rows are balanced by one rule.
template <int TILE_, int STEP_, bool KEYS_>
struct Cut {
    static constexpr int TILE = TILE_, STEP = STEP_;      // stationary rows of a tile, rows of a step: powers of two
    static constexpr bool KEYS = KEYS_;                   // the keys are stationary

    static __device__ __forceinline__ int rows(const AttnParams& p, const Segment& g) { return KEYS ? g.nk : g.nq * p.group; }
    static __device__ __forceinline__ int tiles(const AttnParams& p, const Segment& g) {
        const int n = rows(p, g);
        return n / TILE + (n % TILE != 0);
    }
    // steps of tile t; one (in which nothing is read) where there is nothing on the other side, so that empty rows are written
    static __device__ __forceinline__ int steps(const AttnParams& p, const Segment& g, int t) {
        int n;
        if (KEYS) n = g.nq * p.group;
        else if (!p.causal) n = g.nk;
        else n = keys_of_row(p, g, (min((t + 1) * TILE, g.nq * p.group) - 1) / p.group);
        return max(n / STEP + (n % STEP != 0), 1);
    }
    // units of a kv head
    static __device__ __forceinline__ long long units(const AttnParams& p, const Segment& g) {
        const int n = tiles(p, g);
        if (KEYS || !p.causal) return n ? (long long)n * steps(p, g, 0) : 0;
        long long sum = 0;
        for (int t = 0; t < n; ++t) sum += steps(p, g, t);
        return sum;
    }
};

__device__ __forceinline__ long long warp_total(long long v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ long long warp_running(long long v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(~0u, v, o);
        if ((int)(threadIdx.x % 32) >= o) v += u;
    }
    return v;
}
// a / b for 0 <= a, 0 < b; the short division where both are short
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return (a | b) >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}

// A block's way through its piece of the line: one tile, or a part of one, after the other.
template <typename C>
struct Walker {
    Segment g;
    int s, h, t;                // segment, kv head, tile
    int steps, i0, i1;          // steps of the tile, and which of them are this block's
    long long left;             // units behind this item
    long long units, blocks;    // of the whole line: units, and blocks that share them

    __device__ __forceinline__ void open(const AttnParams& p) {
        steps = C::steps(p, g, t);
        i1 = (int)min((long long)steps, i0 + left);
        left -= i1 - i0;
    }
    __device__ __forceinline__ long long first_unit(long long block) const { return quotient(block * units, blocks); }

    // The piece of block `block` of `grid`, by a warp with all its lanes; of few units every one has a block of its own (two units a block:
    // a single token on 777 keys 14.2 us on the device instead of 11.0).  unit_start: units in front of every segment; NULL (few segments, few tiles): they are counted here.
    // false: nothing to do.
    __device__ __forceinline__ bool begin(const AttnParams& p, const long long* unit_start, int block, int grid) {
        const int lane = threadIdx.x % 32;
        if (unit_start) units = unit_start[p.n_seg];
        else {
            units = 0;
            for (int k = 0; k < p.n_seg; k += 32) units += k + lane < p.n_seg ? C::units(p, segment_of(p, k + lane)) * p.kv_heads : 0;
            units = warp_total(units);
        }
        blocks = min((long long)grid, max(units, 1LL));
        if (block >= blocks || units == 0) return false;
        long long off = first_unit(block), mine = 0;
        left = first_unit(block + 1) - off;
        if (unit_start) {
            s = last_place(unit_start, p.n_seg, off);           // the last segment that begins at or before this unit
            off -= unit_start[s];
            mine = unit_start[s + 1] - unit_start[s];
        } else {
            for (int k = 0;; k += 32) {
                const long long n = k + lane < p.n_seg ? C::units(p, segment_of(p, k + lane)) * p.kv_heads : 0;
                const long long run = warp_running(n);
                const unsigned beyond = __ballot_sync(~0u, run > off);
                if (beyond) {
                    const int at = __ffs(beyond) - 1;
                    s = k + at;
                    mine = __shfl_sync(~0u, n, at);
                    off -= __shfl_sync(~0u, run, at) - mine;
                    break;
                }
                off -= __shfl_sync(~0u, run, 31);
            }
        }
        g = segment_of(p, s);
        const long long per_head = quotient(mine, p.kv_heads);
        h = (int)quotient(off, per_head);
        off -= h * per_head;
        if (C::KEYS || !p.causal) {
            const int n = C::steps(p, g, 0);
            t = (int)quotient(off, n);
            i0 = (int)(off - (long long)t * n);
        } else {
            const int tiles = C::tiles(p, g);
            for (t = 0;; t += 32) {
                const long long run = warp_running(t + lane < tiles ? C::steps(p, g, t + lane) : 0);
                const unsigned beyond = __ballot_sync(~0u, run > off);
                if (beyond) {
                    const int at = __ffs(beyond) - 1;
                    if (at) off -= __shfl_sync(~0u, run, at - 1);
                    t += at;
                    break;
                }
                off -= __shfl_sync(~0u, run, 31);
            }
            i0 = (int)off;
        }
        open(p);
        return true;
    }
    __device__ __forceinline__ bool next(const AttnParams& p) {
        if (left <= 0) return false;
        i0 = 0;
        if (++t >= C::tiles(p, g)) {
            t = 0;
            if (++h >= p.kv_heads) {
                h = 0;
                do { g = segment_of(p, ++s); } while (C::rows(p, g) == 0);
            }
        }
        open(p);
        return true;
    }
    // after begin(): the block in which this item's tile begins
    __device__ __forceinline__ int first_block(int block) const {
        return (int)quotient((first_unit(block) - i0 + 1) * blocks - 1, units);
    }
};

// unit_start[s]: units in front of segment s.  By one block.
constexpr int PLAN_THREADS = 1024;
template <typename C>
static __device__ void plan_units(const AttnParams& p, long long* unit_start) {
    __shared__ long long totals[PLAN_THREADS / 32];
    long long before = 0;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int s0 = 0; s0 < p.n_seg; s0 += PLAN_THREADS) {
        const int s = s0 + threadIdx.x;
        const long long n = warp_running(s < p.n_seg ? C::units(p, segment_of(p, s)) * p.kv_heads : 0);
        if (lane == 31) totals[warp] = n;
        __syncthreads();
        long long sum = before;
        for (int w = 0; w < PLAN_THREADS / 32; ++w) {
            if (w < warp) sum += totals[w];
            before += totals[w];
        }
        if (s < p.n_seg) unit_start[s + 1] = sum + n;
        __syncthreads();
    }
    if (threadIdx.x == 0) unit_start[0] = 0;
}
// Whether the blocks count the units themselves: a launch less, for a few hundred instructions in every warp.
constexpr int COUNT_SEGMENTS = 256, COUNT_TILES = 64;
static inline bool counts_itself(const AttnParams& p, int tile) {
    return p.n_seg <= COUNT_SEGMENTS && (!p.causal || (long long)p.n_q * p.group <= (long long)COUNT_TILES * tile);
}

// A kernel may start before the one in front of it in the stream has ended; it waits where it first reads what that one wrote.
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... A, typename... B>
static inline cudaError_t launch_after(void (*kernel)(A...), dim3 grid, int threads, size_t smem, cudaStream_t s, B... args) {
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute a{};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &a;
    c.numAttrs = 1;
    note_launch();
    return cudaLaunchKernelEx(&c, kernel, args...);
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
