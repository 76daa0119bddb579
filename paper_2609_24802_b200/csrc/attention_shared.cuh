// Attention over dense and paged relations: what the kernels and the host share.
#pragma once
#include <cuda_bf16.h>
#include <limits.h>
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
    const struct Segment* line;     // shared prefixes: the segments of the line, n_seg of them (NULL: they follow from the arrays above)
    int n_seg, n_q, n_kv, heads, kv_heads, group, D, causal;
    long long n_pages, page_size, table_stride, max_pages, page_stride, slot_stride;
    float scale;
    int item_cost, uneven;          // units that a tile costs beside its steps; whether steps cost several (see Cut)
    int whole_sectors;              // of which outputs 16 features of a row are a whole sector (WHOLE_OUT, ...)
    int kv_box, q_box;              // rows that a box of the tensor maps brings (0: rows are copied one by one)
};

enum { WHOLE_OUT = 1, WHOLE_GQ = 2, WHOLE_GK = 4, WHOLE_GV = 8 };

// A segment's rows [q0, q0 + nq) and its keys [k0, k0 + nk) (paged: k0 = 0), bounds clamped to the arrays.  length: its tokens, of which a
// cache may hold fewer (the rows' positions count from its end, not from that of the table).
struct Segment { int q0, nq, k0, nk, length; };

// Rows and positions end here, so that a tile's last row number fits 32 bits.
constexpr long long MOST_ROWS = 0x7fff0000LL;

__host__ __device__ __forceinline__ int clamp_to(int v, int hi) { return min(max(v, 0), hi); }

// (the bounds of rows and of dense keys: p.q_start and p.kv_start, or a copy of them)
__host__ __device__ __forceinline__ Segment segment_of(const AttnParams& p, int s, const int32_t* q_start, const int32_t* kv_start) {
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
__host__ __device__ __forceinline__ Segment segment_of(const AttnParams& p, int s) { return segment_of(p, s, p.q_start, p.kv_start); }

// keys that row t of the segment's nq rows reads: [0, this)
__host__ __device__ __forceinline__ int keys_of_row(const AttnParams& p, const Segment& g, int t) {
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

// Whether a row of a dense segment reads one key of the first `most` (the segment's rows under the triangle: whether the last of them does,
// then none reads more): its weight is 1 whatever the score, so scores have no gradient.  (Masks of up to 32 keys are counted; where a
// longer one leaves a single key the gradient is what is left of dP - delta, a few 2^-23 of either.)
__device__ __forceinline__ bool reads_one_key(const AttnParams& p, const Segment& g, int most) {
    if (!p.mask || most > 32) return most == 1;
    int n = 0;
    for (int j = 0; j < most; ++j) n += p.mask[g.k0 + j] != 0;
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

// Shared prefixes: the keys of a line's segment begin at position g.k0, key j lies at position (g.k0 & ~31) + j of the sequence whose pages
// row `row` of the table names, and those in front of g.k0 count as masked.  (So groups of 8 to 32 keys stay inside of a page.)
__device__ __forceinline__ Place shared_place(const AttnParams& p, const Segment& g, int row, int j) {
    const int at = (g.k0 & ~31) + j, page = at / (int)p.page_size;
    if (at < g.k0) return {-1, 0};
    const int id = p.table[(long long)row * p.table_stride + page];
    return {id >= p.n_pages ? -1 : id, at - page * (int)p.page_size};
}

// The last of n ascending places that is at most `v`, which start[0] is: by a warp with all its lanes, 32 places a round.
template <typename V>
__device__ __forceinline__ int last_place(const V* start, int n, V v) {
    int lo = 0, hi = n;
    if (n <= 128) {             // few: all at once
        int count = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = 32 * k + (int)(threadIdx.x % 32);
            count += __popc(__ballot_sync(~0u, at < n && start[at] <= v));
        }
        return max(count - 1, 0);
    }
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

// a / b for 0 <= a, 0 < b; the short division where both are short
__host__ __device__ __forceinline__ long long quotient(long long a, long long b) {
    return (a | b) >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}
// the same towards minus infinity, for any a, and towards plus infinity
__host__ __device__ __forceinline__ long long floor_quotient(long long a, long long b) { return a >= 0 ? quotient(a, b) : -quotient(b - 1 - a, b); }
__host__ __device__ __forceinline__ long long ceil_quotient(long long a, long long b) { return -floor_quotient(-a, b); }

// Sum of floor((a k + b) / m) over k in [0, n), for 0 <= a, b: whole multiples of m leave a and b; what remains counts the lattice points
// below a line, which are counted again along the other axis, with a and m exchanged, as in Euclid's algorithm.
__host__ __device__ __forceinline__ long long lattice_points(long long n, long long a, long long b, long long m) {
    long long sum = 0, sign = 1;
    while (n > 0) {
        const long long qa = quotient(a, m), qb = quotient(b, m);
        a -= qa * m;
        b -= qb * m;
        sum += sign * (qa * (n * (n - 1) / 2) + qb * n);
        const long long top = quotient(a * (n - 1) + b, m);         // the value of the last k; value v is reached from k = ceil((v m - b) / a) on
        if (top == 0) break;
        // sum over v in [1, top] of n - ceil((v m - b) / a), with v = w + 1
        sum += sign * n * top;
        sign = -sign;
        const long long nb = m - b + a - 1, nm = a;
        a = m;
        b = nb;
        m = nm;
        n = top;
    }
    return sum;
}

// ---- How the work is cut.  A segment's heads share keys, so the rows of a group's heads are packed: packed row r of a kv head is row
// r / group, head kv_head * group + r % group.  A tile of stationary rows (packed rows, or keys for their gradients) meets the other
// side in steps; a unit is one step of one tile of one kv head.  All units of a call stand in one line (segment, kv head, tile,
// step), and the blocks take equal pieces of it: a piece that begins or ends inside a tile leaves a partial state in the
// workspace, and a last kernel joins those in order.  So short and long, few and many rows are balanced by one rule.
// Beginning and ending a tile takes a block as long as some steps do (about 15000 cycles forward, where a step takes 3700).  Where the
// tiles of a line have all numbers of steps, as under a triangle, equal numbers of steps would give the blocks of its short tiles several
// times the work, so a tile counts item_cost units more, in front of its steps.  Under them nothing is done: a piece that ends there has
// none of the tile, one that begins there has its first step.  Where full tiles stand beside tiles of a few rows, whose steps wait for memory
// (2500 cycles against 3700 at a width of 128, 2360 against 3550 at 64), a step costs two or three units; it is done by the piece that has its last one.
enum CutMode { CUT_STEPS, CUT_COSTS, CUT_LINE };          // units are steps; tiles and steps cost as p says; the same, and p.line has the segments
template <int TILE_, int STEP_, bool KEYS_, int MODE = CUT_STEPS>
struct Cut {
    static constexpr int TILE = TILE_, STEP = STEP_;      // stationary rows of a tile, rows of a step: powers of two
    static constexpr bool KEYS = KEYS_;                   // the keys are stationary
    static constexpr bool PLAIN = MODE == CUT_STEPS;

    static __host__ __device__ __forceinline__ Segment segment(const AttnParams& p, int s) { return MODE == CUT_LINE ? p.line[s] : segment_of(p, s); }
    static __host__ __device__ __forceinline__ int rows(const AttnParams& p, const Segment& g) { return KEYS ? g.nk : g.nq * p.group; }
    static __host__ __device__ __forceinline__ int tiles(const AttnParams& p, const Segment& g) {
        const int n = rows(p, g);
        return n / TILE + (n % TILE != 0);
    }
    // steps in front of a tile's first one (keys stationary, under the triangle: packed rows that read none of its keys)
    static __host__ __device__ __forceinline__ int skipped(const AttnParams& p, const Segment& g, int t) {
        if (!KEYS || !p.causal) return 0;
        const long long first = (long long)t * TILE - (g.length - g.nq);        // the first row that reads the tile's first key
        const int packed = g.nq * p.group;
        return first <= 0 ? 0 : first >= g.nq ? packed / STEP : (int)first * p.group / STEP;
    }
    // steps of tile t; one (in which nothing is read) where there is nothing on the other side, so that empty rows are written
    static __host__ __device__ __forceinline__ int steps(const AttnParams& p, const Segment& g, int t) {
        int n;
        if (KEYS) n = g.nq * p.group;
        else if (!p.causal) n = g.nk;
        else {
            const int packed = g.nq * p.group, end = packed - t * TILE > TILE ? (t + 1) * TILE : packed;
            n = keys_of_row(p, g, (end - 1) / p.group);
        }
        n = n / STEP + (n % STEP != 0) - skipped(p, g, t);
        return n > 1 ? n : 1;
    }
    // Steps of the first t tiles (t <= tiles()).  Under the triangle steps(k) is max(1, floor((x k + y) / z)), cut off at the segment's
    // keys or rows: a sum of floors in the middle.
    static __host__ __device__ __noinline__ long long steps_before(const AttnParams& p, const Segment& g, int t) {
        if (t == 0) return 0;
        if (t == 1 || !p.causal) return (long long)t * steps(p, g, 0);
        const long long c = (long long)g.length - g.nq;
        if (KEYS) {
            if (g.nq == 0) return t;
            static_assert(!KEYS || TILE == STEP, "a tile of keys skips `group` steps more than the one in front of it");
            // skipped(k) = k group + floor(-c group / STEP) from the first tile k0 on that skips any rows; none is skipped in front of it
            const long long total = ceil_quotient((long long)g.nq * p.group, STEP), k0 = c <= 0 ? 0 : ceil_quotient(c, TILE);
            if (t <= k0) return t * total;
            return t * total - p.group * ((t - 1LL) * t / 2 - (k0 - 1) * k0 / 2) - (t - k0) * floor_quotient(-c * p.group, STEP);
        }
        // the last tile apart: its rows may end early.  The others: floor((TILE k + b) / m), the last row of tile k being (TILE k + TILE - 1) / group
        const int last = tiles(p, g) - 1;
        const long long m = (long long)STEP * p.group, b = TILE - 1 + p.group * (c + STEP), most = g.nk ? ceil_quotient(g.nk, STEP) : 1;
        const long long n = t <= last ? t : last;
        const long long lo = ceil_quotient(2 * m - b, TILE), hi = ceil_quotient(most * m - b, TILE);          // from where on there are 2 steps, all steps
        const long long k1 = lo < 0 ? 0 : lo < n ? lo : n, k2 = hi < k1 ? k1 : hi < n ? hi : n;
        return k1 + (k1 < k2 ? lattice_points(k2 - k1, TILE, TILE * k1 + b, m) : 0) + (n - k2) * most + (t > last ? steps(p, g, last) : 0);
    }
    static __host__ __device__ __forceinline__ int item_cost(const AttnParams& p) { return MODE == CUT_STEPS ? 0 : p.item_cost; }
    static __host__ __device__ __forceinline__ bool uneven(const AttnParams& p) { return MODE != CUT_STEPS && p.uneven; }
    static __host__ __device__ __forceinline__ int step_cost(const AttnParams& p, const Segment& g) { return !uneven(p) ? 1 : rows(p, g) <= 128 ? 2 : 3; }
    // units of the first t tiles, and of all tiles of a kv head
    static __host__ __device__ __forceinline__ long long before(const AttnParams& p, const Segment& g, int t) {
        return steps_before(p, g, t) * step_cost(p, g) + (long long)t * item_cost(p);
    }
    static __host__ __device__ __forceinline__ long long units(const AttnParams& p, const Segment& g) {
        if (!PLAIN) return before(p, g, tiles(p, g));
        const int n = tiles(p, g);
        if (KEYS || !p.causal) return n ? (long long)n * steps(p, g, 0) : 0;
        long long sum = 0;
        for (int t = 0; t < n; ++t) sum += steps(p, g, t);
        return sum;
    }
};

// The cut of accumulated weights: of a segment with few packed rows the rows stay, in one tile, and steps are tiles of keys; of more the keys
// stay.
constexpr int WT_TILE = 128;
struct WtCut {
    static constexpr bool PLAIN = false;
    typedef Cut<WT_TILE, WT_TILE, true, CUT_COSTS> Wide;        // (tiles cost nothing)
    static __host__ __device__ __forceinline__ bool narrow(const AttnParams& p, const Segment& g) { return (long long)g.nq * p.group <= WT_TILE; }
    static __host__ __device__ __forceinline__ int rows(const AttnParams&, const Segment& g) { return g.nk; }
    static __host__ __device__ __forceinline__ int tiles(const AttnParams& p, const Segment& g) { return narrow(p, g) ? g.nk > 0 : Wide::tiles(p, g); }
    static __host__ __device__ __forceinline__ int skipped(const AttnParams& p, const Segment& g, int t) { return narrow(p, g) ? 0 : Wide::skipped(p, g, t); }
    static __host__ __device__ __forceinline__ int steps(const AttnParams& p, const Segment& g, int t) { return narrow(p, g) ? Wide::tiles(p, g) : Wide::steps(p, g, t); }
    static __host__ __device__ __forceinline__ Segment segment(const AttnParams& p, int s) { return segment_of(p, s); }
    static __host__ __device__ __forceinline__ int item_cost(const AttnParams&) { return 0; }
    static __host__ __device__ __forceinline__ bool uneven(const AttnParams&) { return false; }
    static __host__ __device__ __forceinline__ int step_cost(const AttnParams&, const Segment&) { return 1; }
    static __host__ __device__ __forceinline__ long long before(const AttnParams& p, const Segment& g, int t) {
        return narrow(p, g) ? (long long)t * Wide::tiles(p, g) : Wide::before(p, g, t);
    }
    static __host__ __device__ __forceinline__ long long units(const AttnParams& p, const Segment& g) { return before(p, g, tiles(p, g)); }
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
// A block's way through its piece of the line: one tile, or a part of one, after the other.
template <typename C>
struct Walker {
    Segment g;
    int s, h, t;                // segment, kv head, tile
    int steps, i0, i1;          // steps of the tile, and which of them are this block's
    long long left;             // units behind this item
    long long units, blocks;    // of the whole line: units, and blocks that share them
    long long start;            // the piece's first unit, counted from the beginning of its tile
    bool here;                  // this block has any

    // the tile's steps from its unit `off` on; false: the piece ends in front of the tile's first step
    __host__ __device__ __forceinline__ bool open(const AttnParams& p, long long off) {
        steps = C::steps(p, g, t);
        if (C::PLAIN) {
            i0 = (int)off;
            i1 = (int)min((long long)steps, i0 + left);
            left -= i1 - i0;
            return true;
        }
        const int cost = C::step_cost(p, g);
        const long long end = min((long long)steps * cost + C::item_cost(p), off + left);
        left -= end - off;
        auto steps_of = [&](long long u) { return u <= 0 ? 0 : cost == 1 ? (int)u : (int)quotient(u, cost); };
        i0 = steps_of(off - C::item_cost(p));
        i1 = steps_of(end - C::item_cost(p));
        return i1 > i0;
    }
    // blocks that take part: every piece has a step's units, so that the blocks between a tile's first and last one all have steps of it
    static __host__ __device__ __forceinline__ long long pieces(const AttnParams& p, long long units, int grid) {
        return min((long long)grid, max(C::uneven(p) ? units / 3 : units, 1LL));
    }
    __host__ __device__ __forceinline__ long long first_unit(long long block) const { return quotient(block * units, blocks); }

    // The piece of block `block` of `grid`, by a warp with all its lanes; of few units every one has a block of its own (two units a block:
    // a single token on 777 keys 14.2 us on the device instead of 11.0).  unit_start: units in front of every segment; NULL (few segments, few tiles): they are counted here.
    // false: nothing to do.
    __device__ __forceinline__ bool begin(const AttnParams& p, const long long* unit_start, int block, int grid) {
        const int lane = threadIdx.x % 32;
        long long first = 0;            // of segment `lane`
        if (unit_start) units = unit_start[p.n_seg];
        else {
            units = 0;
            for (int k = 0; k < p.n_seg; k += 32) {
                const long long n = k + lane < p.n_seg ? C::units(p, C::segment(p, k + lane)) * p.kv_heads : 0;
                if (k == 0) first = n;
                units += n;
            }
            units = warp_total(units);
        }
        blocks = pieces(p, units, grid);
        if (block >= blocks || units == 0) return false;
        long long off = first_unit(block), mine = 0;
        left = first_unit(block + 1) - off;
        if (unit_start) {
            s = last_place(unit_start, p.n_seg, off);           // the last segment that begins at or before this unit
            off -= unit_start[s];
            mine = unit_start[s + 1] - unit_start[s];
        } else {
            for (int k = 0;; k += 32) {
                const long long n = k == 0 ? first : k + lane < p.n_seg ? C::units(p, C::segment(p, k + lane)) * p.kv_heads : 0;
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
        g = C::segment(p, s);
        const long long per_head = quotient(mine, p.kv_heads);
        h = (int)quotient(off, per_head);
        off -= h * per_head;
        if (!p.causal) {
            const long long n = (long long)C::steps(p, g, 0) * C::step_cost(p, g) + C::item_cost(p);
            t = (int)quotient(off, n);
            off -= t * n;
        } else if (C::PLAIN) {
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
        } else {            // the last tile that begins at or before this unit: 32 places a round, the last few tiles one by one
            const int tiles = C::tiles(p, g);
            int hi = tiles;
            long long ahead = 0;            // units in front of tile t
            t = 0;
            while (hi - t > 8) {
                const int gap = (hi - t + 31) / 32, at = t + lane * gap;
                const long long here = at < hi ? C::before(p, g, at) : LLONG_MAX;
                const unsigned before = __ballot_sync(~0u, here <= off) | 1u;
                const int last = 31 - __clz(before);
                ahead = __shfl_sync(~0u, here, last);
                t += last * gap;
                hi = min(hi, t + gap);
            }
            off -= ahead;
            for (; t + 1 < hi; ++t) {
                const long long n = (long long)C::steps(p, g, t) * C::step_cost(p, g) + C::item_cost(p);
                if (off < n) break;
                off -= n;
            }
        }
        start = off;
        return open(p, off);
    }
    // The same by a thread alone, for a plan that does it for all blocks.
    __host__ __device__ __forceinline__ void begin_alone(const AttnParams& p, const long long* unit_start, int block, int grid) {
        auto last = [](int n, auto at_most) {               // the last of n places that is not beyond; place 0 is not
            int lo = 0, hi = n;
            while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (at_most(mid)) lo = mid; else hi = mid; }
            return lo;
        };
        units = unit_start[p.n_seg];
        blocks = pieces(p, units, grid);
        here = false;
        if (block >= blocks || units == 0) return;
        long long off = first_unit(block);
        left = first_unit(block + 1) - off;
        s = last(p.n_seg, [&](int k) { return unit_start[k] <= off; });
        off -= unit_start[s];
        g = C::segment(p, s);
        const long long per_head = quotient(unit_start[s + 1] - unit_start[s], p.kv_heads);
        h = (int)quotient(off, per_head);
        off -= h * per_head;
        t = last(C::tiles(p, g), [&](int k) { return C::before(p, g, k) <= off; });
        off -= C::before(p, g, t);
        start = off;
        here = open(p, off);
    }
    __host__ __device__ __forceinline__ bool next(const AttnParams& p) {
        if (left <= 0) return false;
        if (++t >= C::tiles(p, g)) {
            t = 0;
            if (++h >= p.kv_heads) {
                h = 0;
                do { g = C::segment(p, ++s); } while (C::rows(p, g) == 0);
            }
        }
        return open(p, 0);
    }
    // after begin() inside of a tile's steps: the block that has its first step
    __host__ __device__ __forceinline__ int first_block(const AttnParams& p, int block) const {
        if (C::PLAIN) return (int)quotient((first_unit(block) - i0 + 1) * blocks - 1, units);
        return (int)quotient((first_unit(block) - start + C::item_cost(p) + C::step_cost(p, g)) * blocks - 1, units);
    }
    // The same of any tile, and how many blocks have steps of it: those with the last unit of its first and of its last step.  begin: the units in
    // front of the segment.
    struct Blocks { int first, parts; };
    static __host__ __device__ __forceinline__ Blocks blocks_of_tile(const AttnParams& p, const Segment& g, long long begin, int h, int t, long long units, long long blocks) {
        const long long start = begin + h * C::units(p, g) + C::before(p, g, t) + C::item_cost(p) - 1;
        const int cost = C::step_cost(p, g);
        auto block_of = [&](long long unit) { return (int)quotient((unit + 1) * blocks - 1, units); };
        const int first = block_of(start + cost);
        return {first, block_of(start + (long long)cost * C::steps(p, g, t)) - first + 1};
    }
};

// The beginning of a block's piece, out of line: the closed forms want many registers for a moment, which inlined were spilled from the loops
// of the other warps (chunk of 2048 on 16384: 559 us instead of 510).  Plain cuts, whose chunks have few tiles, go through them and stay
// inline, as even the call cost 2 %.
template <typename C>
static __device__ __noinline__ void walk_begin(Walker<C>* to, const AttnParams& p, const long long* unit_start, int block, int grid) {
    Walker<C> w{};
    w.here = w.begin(p, unit_start, block, grid);
    if (threadIdx.x % 32 == 0) *to = w;
}

// unit_start[s]: units in front of segment s.  By one block.
constexpr int PLAN_THREADS = 1024;
template <typename C>
static __device__ void plan_units(const AttnParams& p, long long* unit_start) {
    __shared__ long long totals[PLAN_THREADS / 32];
    long long before = 0;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int s0 = 0; s0 < p.n_seg; s0 += PLAN_THREADS) {
        const int s = s0 + threadIdx.x;
        const long long n = warp_running(s < p.n_seg ? C::units(p, C::segment(p, s)) * p.kv_heads : 0);
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
static inline bool counts_itself(const AttnParams& p, int tile, bool closed_form) {
    return p.n_seg <= COUNT_SEGMENTS && (closed_form || !p.causal || (long long)p.n_q * p.group <= (long long)COUNT_TILES * tile);
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

// ---- The preparation of the backward pass: blocks by the work there may be, `rows` rows of `lanes` threads.
constexpr int FEW_KEYS = 16;                            // up to so many keys a row's delta is summed over them
constexpr int PREP_THREADS = 256, PREP_BLOCKS = 4;      // of an SM
// Little work is done by one block, which clears the words for its maxima itself: a launch less (about 5 us of the host's time against
// 1 us for each 256 rows of 64 features).
constexpr int PREP_ALONE = 16;                          // blocks of work
// Under the triangle: looks for rows of few keys, one for each such row that a segment may have and as many of its heads as a warp takes at a
// time.  They are work of their own, as segments may be empty (125 rows in 10000 segments, 2 heads of 64: 5150 us of one block's, now 72; 4 or 64
// looks to a block 72 too, but 16 segments of 20 rows 43 and 42 instead of 41).
constexpr int LOOKS_OF_A_BLOCK = 16;
static __host__ __device__ __forceinline__ long long looks_for_few_keys(const AttnParams& p, int lanes) {
    return p.causal ? (long long)p.n_seg * FEW_KEYS * ((p.heads * lanes + 31) / 32) : 0;
}
static inline long long prepare_blocks(const AttnParams& p, long long rows, int lanes, int sms) {
    const long long n = (rows * lanes + PREP_THREADS - 1) / PREP_THREADS + looks_for_few_keys(p, lanes) / LOOKS_OF_A_BLOCK;
    return n <= PREP_ALONE ? 1 : n < PREP_BLOCKS * sms ? n : PREP_BLOCKS * sms;
}

constexpr int MAX_SMS = 160;            // blocks that workspaces provide for
// Workspaces come on a boundary of 16 bytes; states are put aside in sectors of 32.  (Their sizes have 256 bytes to spare.)
static inline void* on_sectors(void* ws) { return reinterpret_cast<void*>(align_up(reinterpret_cast<uintptr_t>(ws), 256)); }

// Sequences whose caches begin with the same pages: those of group g, [group_start[g], group_start[g + 1]), share positions [0, shared[g]).
struct Prefixes { const int32_t *group_start, *shared; int n_groups; };

size_t attention_shared_bytes(const AttnParams& p, int n_groups);
tiga_status attention_shared(const AttnParams& p, const Prefixes& g, bool bf16, void* ws, cudaStream_t s);
size_t attention_forward_bytes(const AttnParams& p);
size_t attention_backward_bytes(const AttnParams& p);
tiga_status attention_backward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s);
tiga_status attention_forward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s);

// host checks of the descriptors (attention.cu)
tiga_status attention_heads_check(const tiga_heads* h);
tiga_status attention_pages_check(const tiga_pages* c);
tiga_status attention_paged_check(const tiga_pages* c, const tiga_heads* h, int64_t n_q, AttnParams* p);
bool attention_bad_ints(const void* p);
bool attention_bad_weights(const tiga_weights* a);
bool attention_weights_overlap(const tiga_weights* a, int64_t n_seg, int64_t kv_heads);
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
