// Gradients of the online-softmax reducer over dense relations, on the fifth-generation tensor cores.
#include "attention_tiles.cuh"

namespace tiga {

// Two passes of one form, by blocks of their own in one launch (keys first; a pass's blocks share its work).  A block keeps a stationary tile of 128 rows of two arrays, X1 and X2, and goes through the other side in
// steps of 128 rows of Y1 and Y2:
//     keys and values:  X = (key, value), Y = (q, grad_out):   S = X1 Y1^T, dP = X2 Y2^T (both transposed), grad_value += P Y2,
//                                                               grad_key += dS Y1;      all heads of a group pass by: their sum
//     queries:          X = (q, grad_out), Y = (key, value):   S = X1 Y1^T, dP = X2 Y2^T, grad_q += dS Y1
// with P = exp2(S - lse) and dS = P (dP - delta).  Seven products instead of the five of one kernel that adds grad_q up in memory:
// the sums stay in tensor memory, in one order, so results are reproducible, and no fp32 gradient is written and read again.
// P lies over S and dS over dP in 16 bits (tensor memory: 128 + 128 + 2 * 128 columns, all there is).  The products run in two
// streams that take turns: while the threads turn S into P, dP and the last step's grad_key are formed; while they turn dP into dS,
// grad_value and the next step's S.
// A step of 128 lasts about 3480 cycles (products 2048 or 1536, exponentials 1024, the threads' two turns 2200): 4 segments of 4096 rows
// and keys, 16/4 heads of 128, bf16: 1.70 ms alone for both passes.
// fp16: P carries 2^14 and dS a power of two from the largest norms of the segment's rows of grad_out and value, which bound |dP - delta|:
// the largest value cannot overflow, the smallest keep as many digits as there are.
constexpr int BWD_WEIGHT_WARPS = 16, BWD_PRODUCER = BWD_WEIGHT_WARPS, BWD_MMA = BWD_PRODUCER + 4, BWD_WALKER = BWD_MMA + 1;
constexpr int BWD_THREADS = 32 * (BWD_WALKER + 1), BWD_ROWS = 128, BWD_STEP = 128;
template <bool KV, bool CAUSAL> using BwdCut = Cut<BWD_ROWS, BWD_STEP, KV, CAUSAL ? CUT_COSTS : CUT_STEPS>;
template <int DP> struct Bwd {
    static constexpr int TILE = 128 * DP * 2;
    static constexpr int SLOTS = DP == 128 ? 5 : 8;         // tiles of the ring, in the order Y1 Y2 Y1 Y2 ...
    // Entries of what goes along with a step's rows.  Step n's is written once there is room for its Y2, the tile 2 n + 1: then the tile
    // 2 n + 1 - SLOTS is done with.  Of five slots that is Y1 of step n - 2, whose last product comes after all that its step reads: two
    // entries do.  Of eight it is Y2 of step n - 4, so step n - 4 may still read: eight do.
    static constexpr int AUX = DP == 128 ? 2 : 8;
    static constexpr int CONTROL = (2 + SLOTS) * TILE;
    static constexpr int SMEM = CONTROL + (DP == 128 ? 3 : 10) * 1024;
};

template <int AUX, typename C> struct BwdControl {
    unsigned long long full[8], empty[8], aux_full[AUX], x_full, x_empty, s_full, dp_full, p_full, ds_full, acc_full, acc_empty, drain;
    ItemRing items;
    Walker<C> walk;
    uint32_t tmem, abort_word;
    alignas(16) float minus_lse[AUX][BWD_STEP], minus_delta[AUX][BWD_STEP];     // keys stationary: of the step's rows
    uint32_t mask[AUX][4];                                                      // queries stationary: the step's keys
};
static_assert(sizeof(BwdControl<2, BwdCut<true, true>>) <= 3 * 1024 && sizeof(BwdControl<8, BwdCut<true, true>>) <= 10 * 1024, "control block");

struct BwdWork {
    long long *kv_start_unit, *q_start_unit;        // NULL: the blocks count for themselves
    float2* stats;                  // [n_q, heads]: lse in log2 (+inf: the row reads nothing), delta
    uint32_t* norms;                // [n_seg][2], fp16: largest squared norms of a segment's rows of grad_out and value, as bits
    Joint *kv_joints, *q_joints;    // [blocks of the side]
    float *kv_part, *q_part;        // [2 * blocks of the side][rows][gradients of the side][DP]
    int kv_rows, q_rows;            // rows that a partial state holds at most
};

// the power of two that dS of segment s carries (fp16)
__device__ __forceinline__ float gradient_factor(const uint32_t* norms, int s) {
    const uint2 n = reinterpret_cast<const uint2*>(norms)[s];
    const float largest = 2.f * sqrtf(__uint_as_float(n.x)) * sqrtf(__uint_as_float(n.y));
    if (!(largest > 1e-30f && largest < 1e30f)) return 1.f;
    return exp2f(14.f - (float)(ilogbf(largest) + 1));
}

// delta, lse in log2, and the norms behind gradient_factor: a row by LANES threads, 8 features each.  Bound by memory: grad_out and out
// are read once (fp16: value too).  A block has rows that follow one another, so that it passes through their segments in order.  Of few
// keys delta is summed as sum p dP: out is then as large as the values, and its rounding would show in dP - delta (over n keys it is
// smaller by the root of n).
template <typename T>
__device__ __forceinline__ float dot8(const uint4& a, const uint4& b) {
    const T* x = reinterpret_cast<const T*>(&a);
    const T* y = reinterpret_cast<const T*>(&b);
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) d += Half<T>::to(x[e]) * Half<T>::to(y[e]);
    return d;
}
// The largest norm of a segment, as far as this thread's rows go, to memory: a maximum does not depend on the order.
__device__ __forceinline__ void put_norm(uint32_t* norm, float top) {
    const uint32_t bits = __float_as_uint(top);
    if (bits > *(volatile uint32_t*)norm) atomicMax(norm, bits);
}
// ... at the end of a block's rows: once for all of them where they lie in one segment
template <int LANES>
__device__ __forceinline__ void put_last_norms(uint32_t* norms, int s, int first_s, float top) {
    __shared__ uint32_t tops[PREP_THREADS / 32];
    if (__syncthreads_and(s == first_s)) {
        const uint32_t bits = __reduce_max_sync(~0u, __float_as_uint(top));
        if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = bits;
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t most = 0;
            for (int k = 0; k < PREP_THREADS / 32; ++k) most = max(most, tops[k]);
            put_norm(norms + 2LL * s, __uint_as_float(most));
        }
    } else if (threadIdx.x % LANES == 0) put_norm(norms + 2LL * s, top);
}
// Row and head of numbers that grow by one step after the other.  (With divisions for each of them the kernel took 33 us of 163840 rows of
// queries and 240000 of values, fp16, width 64; now 22.)
struct RowHead {
    int row, head, rows, heads, of;         // rows, heads: of a step
    __device__ __forceinline__ RowHead(long long r, int step, int n) : of(n) {
        row = (int)quotient(r, n);
        head = (int)(r - (long long)row * n);
        rows = step / n;
        heads = step - rows * n;
    }
    __device__ __forceinline__ void go_on() {
        row += rows;
        head += heads;
        if (head >= of) { head -= of; ++row; }
    }
};
template <typename T, int LANES>
__global__ void __launch_bounds__(PREP_THREADS, PREP_BLOCKS) attention_prepare_kernel(const AttnParams p, const BwdWork w, const int q_blocks, const int v_blocks) {
    constexpr bool NORMS = operand_type<T>() == 0;
    constexpr int ROWS = PREP_THREADS / LANES;
    wait_for_previous_kernel();
    let_next_kernel_start();
    if (NORMS && gridDim.x == 1) {
        for (int i = threadIdx.x; i < 2 * p.n_seg; i += PREP_THREADS) w.norms[i] = 0;
        __syncthreads();
    }
    // the bounds of few segments at once, so that no look-up waits for the one before it
    __shared__ int32_t bounds[2][PREP_THREADS];
    const int32_t *q_start = p.q_start, *kv_start = p.kv_start;
    if (p.n_seg < PREP_THREADS) {
        if ((int)threadIdx.x <= p.n_seg) { bounds[0][threadIdx.x] = q_start[threadIdx.x]; bounds[1][threadIdx.x] = kv_start[threadIdx.x]; }
        __syncthreads();
        q_start = bounds[0];
        kv_start = bounds[1];
    }
    const int lane = threadIdx.x % LANES;
    const bool in_width = lane * 8 < p.D;
    auto fold = [&](float v) {
#pragma unroll
        for (int d = LANES / 2; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
        return v;
    };
    // the first blocks have rows of queries, the last ones of values (one block: both); where those of a block among `blocks` begin
    const int v_block = (int)blockIdx.x - ((int)gridDim.x - v_blocks);
    auto piece_begin = [&](long long n, int block, int blocks) { return min(quotient(n + (long long)blocks * ROWS - 1, (long long)blocks * ROWS) * ROWS * block, n); };
    const int q_first = clamp_to(q_start[0], p.n_q), q_end = max(clamp_to(q_start[p.n_seg], p.n_q), q_first);
    const long long q_rows = (long long)(q_end - q_first) * p.heads, q_from = piece_begin(q_rows, blockIdx.x, q_blocks), q_to = piece_begin(q_rows, blockIdx.x + 1, q_blocks);
    if (q_from < q_to) {
        Along at_seg;
        at_seg.open(q_start, p.n_seg, q_first + (int)quotient(q_from, p.heads));
        const int first_s = at_seg.s;
        Segment g = segment_of(p, first_s, q_start, kv_start);
        float top = 0.f;
        RowHead here(q_from + threadIdx.x / LANES, ROWS, p.heads);
        for (long long r0 = q_from; r0 < q_to; r0 += ROWS, here.go_on()) {          // whole warps stay together
            const long long r = r0 + threadIdx.x / LANES, row = q_first + here.row, at = row * p.heads + here.head;
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            float lse = 0.f;
            int few = 0;
            bool later = false;
            if (r < q_to) {
                if (in_width) {
                    a = *reinterpret_cast<const uint4*>((const T*)p.go + row * p.go_row + here.head * p.go_head + lane * 8);
                    b = *reinterpret_cast<const uint4*>((const T*)p.o + at * p.D + lane * 8);
                }
                lse = p.lse_in[at];
                const int before = at_seg.s;
                if (at_seg.go_on(q_start, p.n_seg, (int)row)) {
                    if (NORMS && lane == 0) put_norm(w.norms + 2LL * before, top);
                    top = 0.f;
                    g = segment_of(p, at_seg.s, q_start, kv_start);
                }
                if (p.causal) {
                    const int n = keys_of_row(p, g, (int)row - g.q0);
                    later = n > 0 && n <= FEW_KEYS;
                }
                else if (g.nk <= FEW_KEYS && lse != -INFINITY) few = g.nk;
            }
            float dot = fold(dot8<T>(a, b));
            const float norm = NORMS ? fold(dot8<T>(a, a)) : 0.f;
            const int most = __reduce_max_sync(~0u, few);
            if (most) {                     // (whole warps: rows of other segments take part with nothing)
                const int kv_head = here.head / p.group;
                uint4 q = make_uint4(0, 0, 0, 0);
                if (few && in_width) q = *reinterpret_cast<const uint4*>((const T*)p.q + row * p.q_row + here.head * p.q_head + lane * 8);
                float sum = 0.f;
                for (int j = 0; j < most; ++j) {
                    const Place at_key = j < few ? key_place(p, g, at_seg.s, j) : Place{-1, 0};
                    uint4 k = make_uint4(0, 0, 0, 0), v = k;
                    if (at_key.at >= 0 && in_width) {
                        k = *reinterpret_cast<const uint4*>((const T*)p.k + key_offset(p, at_key, kv_head) + lane * 8);
                        v = *reinterpret_cast<const uint4*>((const T*)p.v + value_offset(p, at_key, kv_head) + lane * 8);
                    }
                    const float score = fold(dot8<T>(q, k)), dp = fold(dot8<T>(a, v));
                    if (at_key.at >= 0) sum += ex2((score * p.scale - lse) * LOG2E_F) * dp;
                }
                if (few) dot = sum;
            }
            if (r >= q_to) continue;
            const bool reads = lse != -INFINITY;
            if (lane == 0 && !later) w.stats[at] = make_float2(reads ? lse * LOG2E_F : INFINITY, reads ? dot : 0.f);
            if (NORMS && reads) top = norm == norm ? fmaxf(top, norm) : INFINITY;
        }
        if (NORMS) put_last_norms<LANES>(w.norms, at_seg.s, first_s, top);
    }
    if (NORMS && v_block >= 0) {
        const int k_first = clamp_to(kv_start[0], p.n_kv), k_end = max(clamp_to(kv_start[p.n_seg], p.n_kv), k_first);
        const long long v_rows = (long long)(k_end - k_first) * p.kv_heads, v_from = piece_begin(v_rows, v_block, v_blocks), v_to = piece_begin(v_rows, v_block + 1, v_blocks);
        if (v_from < v_to) {
            Along at_seg;
            at_seg.open(kv_start, p.n_seg, k_first + (int)quotient(v_from, p.kv_heads));
            const int first_s = at_seg.s;
            bool read = segment_of(p, first_s, q_start, kv_start).nq > 0;       // (what no row reads sets no scale)
            float top = 0.f;
            constexpr int AHEAD = 4;            // rows of a thread under way
            RowHead here(v_from + threadIdx.x / LANES, ROWS, p.kv_heads);
            for (long long r0 = v_from; r0 < v_to; r0 += AHEAD * ROWS) {
                uint4 a[AHEAD];
                int rows[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k, here.go_on()) {
                    rows[k] = r0 + k * ROWS + threadIdx.x / LANES < v_to ? k_first + here.row : -1;
                    a[k] = make_uint4(0, 0, 0, 0);
                    if (rows[k] >= 0 && in_width && (!p.mask || p.mask[rows[k]]))
                        a[k] = *reinterpret_cast<const uint4*>((const T*)p.v + rows[k] * p.v_row + here.head * p.v_head + lane * 8);
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const float norm = fold(dot8<T>(a[k], a[k]));
                    if (rows[k] < 0) continue;
                    const int before = at_seg.s;
                    if (at_seg.go_on(kv_start, p.n_seg, rows[k])) {
                        if (lane == 0) put_norm(w.norms + 2LL * before + 1, top);
                        top = 0.f;
                        read = segment_of(p, at_seg.s, q_start, kv_start).nq > 0;
                    }
                    if (read) top = norm == norm ? fmaxf(top, norm) : INFINITY;
                }
            }
            put_last_norms<LANES>(w.norms + 1, at_seg.s, first_s, top);
        }
    }
    if (p.causal) {
        // The rows of few keys are the first ones of every segment, one behind the other: dealt out to all warps of the grid, a row and some of its
        // heads at a time (in the loop above their block was the last to end, by 30 us).
        constexpr int HEADS = 32 / LANES;
        const int pieces = (p.heads + HEADS - 1) / HEADS;
        const long long tasks = looks_for_few_keys(p, LANES), stride = (long long)gridDim.x * (PREP_THREADS / 32);
        for (long long task = (long long)blockIdx.x * (PREP_THREADS / 32) + threadIdx.x / 32; task < tasks; task += stride) {
            const long long of_row = quotient(task, pieces);
            const int s = (int)(of_row / FEW_KEYS), n = (int)(of_row % FEW_KEYS) + 1, head = (int)(task - of_row * pieces) * HEADS + (int)(threadIdx.x % 32) / LANES;
            const Segment g = segment_of(p, s, q_start, kv_start);
            const int t = n - 1 - (g.length - g.nq), row = g.q0 + t;            // the row that reads n keys
            if (t < 0 || t >= g.nq || n > g.nk) continue;
            const bool on = head < p.heads;
            const int kv_head = on ? head / p.group : 0;
            const long long at = (long long)row * p.heads + head;
            const float lse = on ? p.lse_in[at] : -INFINITY;
            uint4 q = make_uint4(0, 0, 0, 0), a = q;
            if (on && in_width) {
                q = *reinterpret_cast<const uint4*>((const T*)p.q + row * p.q_row + head * p.q_head + lane * 8);
                a = *reinterpret_cast<const uint4*>((const T*)p.go + row * p.go_row + head * p.go_head + lane * 8);
            }
            float sum = 0.f;
#pragma unroll 4
            for (int j = 0; j < n; ++j) {               // (masked keys are loaded as well, so that no load waits for the mask)
                uint4 k = make_uint4(0, 0, 0, 0), v = k;
                const Place at_key = {g.k0 + j, 0};
                const bool read = !p.mask || p.mask[at_key.at];
                if (in_width) {
                    k = *reinterpret_cast<const uint4*>((const T*)p.k + key_offset(p, at_key, kv_head) + lane * 8);
                    v = *reinterpret_cast<const uint4*>((const T*)p.v + value_offset(p, at_key, kv_head) + lane * 8);
                }
                const float score = fold(dot8<T>(q, k)), dp = fold(dot8<T>(a, v));
                if (read) sum += ex2((score * p.scale - lse) * LOG2E_F) * dp;
            }
            const bool reads = lse != -INFINITY;
            if (on && lane == 0) w.stats[at] = make_float2(reads ? lse * LOG2E_F : INFINITY, reads ? sum : 0.f);
        }
    }
}

template <typename T, int DP, bool KV, bool CAUSAL>
__device__ __forceinline__ void backward_pass(const AttnParams& p, const BwdWork& w, const TileMaps& maps, const int block, const int blocks) {
    typedef Bwd<DP> C;
    typedef BwdCut<KV, CAUSAL> WorkCut;
    constexpr bool F16 = operand_type<T>() == 0;
    constexpr float BIAS = F16 ? 14.f : 0.f;
    extern __shared__ __align__(1024) unsigned char smem[];
    BwdControl<C::AUX, WorkCut>& ctl = *reinterpret_cast<BwdControl<C::AUX, WorkCut>*>(smem + C::CONTROL);
    const uint32_t x_tile = smem_u32(smem), ring = x_tile + 2 * C::TILE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile uint32_t* abort_word = &ctl.abort_word;
    auto bar = [&](unsigned long long& b) { return smem_u32(&b); };

    wait_for_previous_kernel();
    let_next_kernel_start();
    if (threadIdx.x == 0) {
        items_init(ctl.items, BWD_WALKER);
        for (int i = 0; i < C::SLOTS; ++i) { mbar_init(bar(ctl.full[i]), 128); mbar_init(bar(ctl.empty[i]), 1); }
        for (int i = 0; i < C::AUX; ++i) mbar_init(bar(ctl.aux_full[i]), 4);
        mbar_init(bar(ctl.x_full), 256);
        mbar_init(bar(ctl.x_empty), 1);
        mbar_init(bar(ctl.s_full), 1);
        mbar_init(bar(ctl.dp_full), 1);
        mbar_init(bar(ctl.p_full), 32 * BWD_WEIGHT_WARPS);
        mbar_init(bar(ctl.ds_full), 32 * BWD_WEIGHT_WARPS);
        mbar_init(bar(ctl.acc_full), 1);
        mbar_init(bar(ctl.acc_empty), 32 * BWD_WEIGHT_WARPS);
        mbar_init(bar(ctl.drain), 1);
        ctl.abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    Walker<WorkCut> walk;
    const long long* unit_start = KV ? w.kv_start_unit : w.q_start_unit;
    if (CAUSAL) { if (warp == BWD_WALKER) walk_begin(&ctl.walk, p, unit_start, block, blocks); }
    else {
        walk.here = false;
        if (warp == BWD_WALKER) walk.here = walk.begin(p, unit_start, block, blocks);
    }
    if (warp == BWD_MMA) tmem_alloc(smem_u32(&ctl.tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = ctl.tmem;
    const uint32_t s_at = tmem, dp_at = tmem + 128, acc1 = tmem + 256, acc2 = tmem + 384;

    if (warp == BWD_WALKER) {
        if (lane == 0) {
            if (CAUSAL) walk = ctl.walk;
            (KV ? w.kv_joints : w.q_joints)[block] = joint_of(p, walk, walk.here, block);
            int of = -1;
            float factor = 1.f;
            auto factor_of = [&](int s) {
                if (F16 && s != of) factor = gradient_factor(w.norms, of = s);
                return factor;
            };
            items_hand_out(ctl.items, p, walk, walk.here, A_MINUTE, factor_of);
        }
        __syncwarp();
    } else if (warp >= BWD_PRODUCER && warp < BWD_MMA) {
        // ---------------------------------------------------------------- producers
        const int pw = warp - BWD_PRODUCER;
        uint32_t tiles = 0, steps = 0, items = 0;
        bool ok = true;
        auto wait = [&](unsigned long long& b, uint32_t parity) { return ok = __all_sync(~0u, mbar_wait(bar(b), parity & 1, abort_word)); };
        auto slot_free = [&]() { return tiles < (uint32_t)C::SLOTS || wait(ctl.empty[tiles % C::SLOTS], tiles / C::SLOTS + 1); };
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const Segment g = e.segment();
            const int packed_rows = g.nq * p.group, skip = CAUSAL ? WorkCut::skipped(p, g, e.t) : 0, i0 = e.i0 + skip, i1 = ok ? e.i1 + skip : i0, h = e.h;
            // a row of the other side, or of the tile itself: where key r lies, or whether packed row r is wanted
            Place at;
            bool on;
            float2 stat;
            auto look = [&](bool keys, int r) {
                at = {-1, 0};
                on = false;
                stat = make_float2(INFINITY, 0.f);
                if (keys) {
                    if (r < g.nk && g.nq) at = key_place(p, g, e.s, r);     // (keys that no row reads stay out of the products as masked ones do)
                } else if (r < packed_rows) {
                    const PackedRow pr = packed_row(p, g, h, r);
                    stat = w.stats[(long long)pr.row * p.heads + pr.head];
                    on = stat.x != INFINITY;            // a row that reads nothing: whatever lies there stays out of the products
                }
            };
            auto fetch = [&](uint32_t tile, uint32_t full, bool keys, bool second, Place a, bool wanted, int r) {
                if (keys) fetch_keys<DP>(tile, 32 * pw, full, p, maps, second, a, h, w.stats);
                else fetch_packed<DP>(tile, 32 * pw, full, p, g, maps, second, h, r, wanted, w.stats);
            };
            if (ok && items) wait(ctl.x_empty, items - 1);
            const int x_row = e.t * BWD_ROWS + 32 * pw + lane;
            if (ok) {
                look(KV, x_row);
                for (int y = 0; y < 2; ++y) fetch(x_tile + y * C::TILE, bar(ctl.x_full), KV, y, at, on, x_row);
                ++items;
                look(!KV, i0 * BWD_STEP + 32 * pw + lane);
            }
            for (int i = i0; i < i1 && ok; ++i, ++steps) {
                const Place here = at;
                const bool wanted = on;
                const float2 st = stat;
                const int aux = steps % C::AUX, r = i * BWD_STEP + 32 * pw + lane;
                if (!slot_free()) break;
                fetch(ring + (tiles % C::SLOTS) * C::TILE, bar(ctl.full[tiles % C::SLOTS]), !KV, false, here, wanted, r);
                ++tiles;
                if (!slot_free()) break;
                fetch(ring + (tiles % C::SLOTS) * C::TILE, bar(ctl.full[tiles % C::SLOTS]), !KV, true, here, wanted, r);
                ++tiles;
                if (KV) {
                    ctl.minus_lse[aux][32 * pw + lane] = BIAS - st.x;
                    ctl.minus_delta[aux][32 * pw + lane] = -st.y;
                } else {
                    const uint32_t valid = __ballot_sync(~0u, here.at >= 0);
                    if (lane == 0) ctl.mask[aux][pw] = valid;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.aux_full[aux]));
                if (i + 1 < i1) look(!KV, r + BWD_STEP);
            }
            item_return(ctl.items, item);
        }
        cp_async_wait_all();
        if (*abort_word) {          // boxes may still be on their way: their tiles, as far as they were asked for
            for (uint32_t k = tiles < (uint32_t)C::SLOTS ? 0 : tiles - C::SLOTS; k < tiles; ++k) mbar_wait_for(bar(ctl.full[k % C::SLOTS]), (k / C::SLOTS) & 1, HALF_A_SECOND);
            if (items) mbar_wait_for(bar(ctl.x_full), (items - 1) & 1, HALF_A_SECOND);
        }
    } else if (warp == BWD_MMA) {
        // ---------------------------------------------------------------- matrix instructions
        // the warp goes its way together, one thread issues
        const uint32_t s_shape = mma_shape<T>(BWD_STEP, false), acc_shape = mma_shape<T>(DP, true);
        const uint32_t sign = p.scale < 0.f ? MMA_NEGATE_A : 0;
        uint32_t tile0 = 0, steps = 0, items = 0;
        bool ok = true;
        // descriptors differ in their address alone (see the forward kernel)
        const uint32_t x_desc = smem_desc(x_tile, 16), inner_desc = smem_desc(ring, 16), outer_desc = smem_desc(ring, 128 * 128);
        auto slot = [&](uint32_t tile) { return (tile % C::SLOTS) * (uint32_t)(C::TILE / 16); };
        auto wait = [&](unsigned long long& b, uint32_t parity) { ok = __all_sync(~0u, ok && mbar_wait(bar(b), parity & 1, abort_word)); };
        auto wait_tile = [&](uint32_t tile) {
            wait(ctl.full[tile % C::SLOTS], tile / C::SLOTS);
            fence_async_proxy();
        };
        auto wait_threads = [&](unsigned long long& b, uint32_t parity) {
            wait(b, parity);
            tmem_fence_after();
        };
        auto commit = [&](unsigned long long& b) { if (elected()) mma_commit(bar(b)); };
        auto release = [&](uint32_t tile) { commit(ctl.empty[tile % C::SLOTS]); };
        // d = X Y^T, features in pieces of 16
        auto inner = [&](uint32_t d, int second, uint32_t tile, uint32_t shape) {
            const uint32_t x = x_desc + second * (C::TILE / 16), y = inner_desc + slot(tile);
            if (elected())
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
                    if (k * 16 < p.D) mma_ss(d, x + piece(k), y + piece(k), shape, k > 0);
            __syncwarp();
        };
        // acc (+)= (16-bit weights at a: 32 of them in the first half of each 32 columns) Y
        auto outer = [&](uint32_t acc, uint32_t a, uint32_t tile, bool add) {
            const uint32_t y = outer_desc + slot(tile);
            if (elected()) {
                mma_ts(acc, a, y, acc_shape, add);
#pragma unroll
                for (int k = 1; k < BWD_STEP / 16; ++k) mma_ts(acc, a + (k / 2) * 32 + (k % 2) * 8, y + k * (2048 / 16), acc_shape, true);
            }
            __syncwarp();
        };
        for (;; ++items) {
            const Item& e = item_take(ctl.items, items);
            if (e.steps == 0) break;
            const int n = e.i1 - e.i0;
            item_return(ctl.items, items);
            wait(ctl.x_full, items);
            wait_tile(tile0);
            if (!ok) continue;
            inner(s_at, 0, tile0, s_shape | sign);
            commit(ctl.s_full);
            wait_tile(tile0 + 1);
            if (!ok) continue;
            inner(dp_at, 1, tile0 + 1, s_shape);
            commit(ctl.dp_full);
            if (!KV) release(tile0 + 1);
            if (n == 1) commit(ctl.x_empty);
            for (int i = 0; i < n; ++i, ++steps) {
                const uint32_t y1 = tile0 + 2 * i, y2 = y1 + 1;
                const bool again = i + 1 < n;
                wait_threads(ctl.p_full, steps);
                if (i == 0 && items) wait(ctl.acc_empty, items - 1);
                if (!ok) break;
                if (KV) {
                    outer(acc2, s_at, y2, i > 0);
                    release(y2);
                }
                if (again) {
                    wait_tile(y1 + 2);
                    if (!ok) break;
                    inner(s_at, 0, y1 + 2, s_shape | sign);
                    commit(ctl.s_full);
                }
                wait_threads(ctl.ds_full, steps);
                if (!ok) break;
                outer(acc1, dp_at, y1, i > 0);
                release(y1);
                if (again) {
                    wait_tile(y2 + 2);
                    if (!ok) break;
                    inner(dp_at, 1, y2 + 2, s_shape);
                    commit(ctl.dp_full);
                    if (!KV) release(y2 + 2);
                    if (i + 2 == n) commit(ctl.x_empty);
                }
            }
            if (!ok) continue;
            commit(ctl.acc_full);
            tile0 += 2 * n;
        }
        commit(ctl.drain);
        mbar_wait_for(bar(ctl.drain), 0, HALF_A_SECOND);
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- weights: warpgroup x has 32 of a step's 128 columns
        const int x = warp / 4;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const int row = threadIdx.x & 127;
        const uint32_t S = s_at + lanes + 32 * x, dP = dp_at + lanes + 32 * x;
        const float scale2 = fmaxf(fabsf(p.scale) * LOG2E_F, 1e-30f);
        const f32x2 sc2 = dup2(scale2);
        uint32_t steps = 0, items = 0;
        bool ok = true;
        for (;; ++items) {
            const Item& item = item_take(ctl.items, items);
            if (item.steps == 0) break;
            const int n = item.i1 - item.i0, r = item.t * BWD_ROWS + row, n_rows = WorkCut::rows(p, item.segment());
            const bool valid = r < n_rows;
            const bool warp_on = (r & ~31) < n_rows;
            const float factor = F16 ? ctl.items.factor[items % ITEMS] : 1.f;
            const f32x2 ds2 = dup2(F16 ? factor * 0x1p-14f : 1.f);
            f32x2 my_lse = 0, my_delta = 0;
            long long out_row = 0;
            bool masked = false;
            int keys = item.nk;             // queries stationary: keys that the row reads
            // under the triangle, from this thread's first column of the item on: columns that are left out (keys stationary: rows in front of
            // the first one that reads the key), or columns that are read (queries stationary)
            int edge = KV ? 0 : INT32_MAX;
            if (KV) {
                out_row = (long long)(item.k0 + r) * p.kv_heads + item.h;
                masked = valid && (item.nq == 0 || key_place(p, item.segment(), item.s, r).at < 0);
                if (CAUSAL && valid) edge = min(max(r - (item.length - item.nq), 0), item.nq) * p.group - (item.i0 + WorkCut::skipped(p, item.segment(), item.t)) * BWD_STEP - 32 * x;
            } else if (valid) {
                const PackedRow pr = packed_row(p, item.segment(), item.h, r);
                if (CAUSAL) keys = keys_of_row(p, item.segment(), pr.row - item.q0);
                if (CAUSAL) edge = keys - item.i0 * BWD_STEP - 32 * x;
                out_row = (long long)pr.row * p.heads + pr.head;
                const float2 st = w.stats[out_row];
                my_lse = dup2(BIAS - st.x);
                my_delta = dup2(-st.y);
                masked = st.x == INFINITY;
            }
            for (int i = 0; i < n; ++i, ++steps) {
                const uint32_t aux = steps % C::AUX;
                ok = ok && mbar_wait(bar(ctl.aux_full[aux]), (steps / C::AUX) & 1, abort_word) && mbar_wait(bar(ctl.s_full), steps & 1, abort_word);
                ok = __all_sync(~0u, ok);
                if (!ok) continue;
                tmem_fence_after();
                f32x2 e[16];
                if (warp_on) {
                    uint32_t v[32];
                    tmem_ld32(S, v);
                    const float4* nl = reinterpret_cast<const float4*>(ctl.minus_lse[aux] + 32 * x);
                    uint32_t keep = KV ? ~0u : ctl.mask[aux][x];
                    if (CAUSAL) {
                        const int at = edge - i * BWD_STEP;
                        keep &= KV ? (at <= 0 ? ~0u : at >= 32 ? 0u : ~0u << at) : at >= 32 ? ~0u : at <= 0 ? 0u : (1u << at) - 1;
                    }
                    const bool whole = CAUSAL ? __all_sync(~0u, keep == ~0u) : keep == ~0u;
                    tmem_wait_ld(v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        f32x2 lse = my_lse;
                        if (KV) { const float4 l4 = nl[k / 2]; lse = k & 1 ? pack2(l4.z, l4.w) : pack2(l4.x, l4.y); }
                        float a, b;
                        unpack2(fma2(pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), sc2, lse), a, b);
                        a = ex2(a);
                        b = ex2(b);
                        if (!whole) {
                            if (!(keep >> (2 * k) & 1)) a = 0.f;
                            if (!(keep >> (2 * k + 1) & 1)) b = 0.f;
                        }
                        e[k] = pack2(a, b);
                        if (KV) v[k] = pack_half<T>(a, b);
                    }
                    if (KV) {
                        tmem_st16(S, v);
                        tmem_wait_st();
                    }
                }
                tmem_fence_before();
                mbar_arrive(bar(ctl.p_full));
                ok = mbar_wait(bar(ctl.dp_full), steps & 1, abort_word);
                ok = __all_sync(~0u, ok);
                if (!ok) continue;
                tmem_fence_after();
                if (warp_on) {
                    uint32_t v[32];
                    tmem_ld32(dP, v);
                    const float4* nd = reinterpret_cast<const float4*>(ctl.minus_delta[aux] + 32 * x);
                    tmem_wait_ld(v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        f32x2 delta = my_delta;
                        if (KV) { const float4 d4 = nd[k / 2]; delta = k & 1 ? pack2(d4.z, d4.w) : pack2(d4.x, d4.y); }
                        f32x2 g = mul2(e[k], add2(pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), delta));
                        if (F16) g = mul2(g, ds2);
                        float a, b;
                        unpack2(g, a, b);
                        v[k] = pack_half<T>(a, b);
                    }
                    tmem_st16(dP, v);
                    tmem_wait_st();
                }
                tmem_fence_before();
                mbar_arrive(bar(ctl.ds_full));
            }
            ok = ok && mbar_wait(bar(ctl.acc_full), items & 1, abort_word);
            ok = __all_sync(~0u, ok);
            tmem_fence_after();
            // keys stationary: warpgroups 0 and 1 write grad_key, 2 and 3 grad_value, a half of the features each; queries: a quarter each
            const bool whole_tile = n == item.steps;
            const int rows = KV ? w.kv_rows : w.q_rows;
            constexpr int SIDES = KV ? 2 : 1, MINE = DP * SIDES / 4;        // this thread's features of a row
            const int side = KV ? x / 2 : 0, f0 = (KV ? x % 2 : x) * MINE;
            const bool zero = masked || (side == 0 && reads_one_key(p, item.segment(), keys));
            const uint32_t acc = (side ? acc2 : acc1) + lanes;
            const float finish = side ? (F16 ? 0x1p-14f : 1.f) : p.scale / factor;
            T* out = (T*)(KV ? (side ? p.gv : p.gk) : p.gq);
            float* part = (KV ? w.kv_part : w.q_part) + ((((2LL * block + (item.i0 == 0)) * rows + row) * SIDES) + side) * DP;
            if (warp_on)
#pragma unroll 1
                for (int f = f0; f < f0 + MINE; f += 16) {
                    uint32_t v[16];
                    tmem_ld16(acc + f, v);
                    tmem_wait_ld(v);
                    if (!ok)
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] = 0x7fffffffu;
                    if (whole_tile) {
                        uint4 o[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t h[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                h[k] = zero && ok ? 0u : pack_half<T>(__uint_as_float(v[8 * c + 2 * k]) * finish, __uint_as_float(v[8 * c + 2 * k + 1]) * finish);
                            o[c] = make_uint4(h[0], h[1], h[2], h[3]);
                        }
                        store_pieces(o, out + out_row * p.D + f, valid && out, (p.D - f) / 8, p.whole_sectors & (KV ? (side ? WHOLE_GV : WHOLE_GK) : WHOLE_GQ));
                    } else if (valid) {
                        store_sector(part + f, v);
                        store_sector(part + f + 8, v + 8);
                    }
                }
            tmem_fence_before();
            mbar_arrive(bar(ctl.acc_empty));
            item_return(ctl.items, items);
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == BWD_MMA) { tmem_fence_after(); tmem_free(tmem, 512); }
}

template <typename T, int DP, bool CAUSAL>
__global__ void __launch_bounds__(BWD_THREADS, 1) attention_backward_kernel(const __grid_constant__ AttnParams p, const BwdWork w, const __grid_constant__ TileMaps maps, const int kv_blocks) {
    if ((int)blockIdx.x < kv_blocks) backward_pass<T, DP, true, CAUSAL>(p, w, maps, blockIdx.x, kv_blocks);
    else backward_pass<T, DP, false, CAUSAL>(p, w, maps, (int)blockIdx.x - kv_blocks, (int)gridDim.x - kv_blocks);
}

// Adds up the partial sums of a tile that several blocks shared, in the order of its steps.  A warp has a row of one gradient; many parts
// (few tiles, a long axis) are shared by the block's warps, whose sums are added in order.
constexpr int SUM_WARPS = 8, SUM_Y = 16, SUM_FEW = 8;

template <typename T, int DP, bool KV>
__device__ __forceinline__ void sum_pass(const AttnParams& p, const BwdWork& w, const int block) {
    typedef BwdCut<KV, false> WorkCut;             // (rows of a tile: the same for all)
    constexpr int SIDES = KV ? 2 : 1, E = DP / 32;
    constexpr bool F16 = operand_type<T>() == 0;
    const Joint& j = (KV ? w.kv_joints : w.q_joints)[block];
    const int parts = j.parts;
    if (parts == 0) return;
    const Item it = j.item;
    const Segment g = it.segment();
    const int first = j.first, rows = min(WorkCut::rows(p, g) - it.t * BWD_ROWS, BWD_ROWS), cap = KV ? w.kv_rows : w.q_rows;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const float factor = F16 ? gradient_factor(w.norms, it.s) : 1.f;
    __shared__ float sh[SUM_WARPS][DP];
    const bool few = parts <= SUM_FEW;
    for (int rs = few ? blockIdx.y * SUM_WARPS + warp : blockIdx.y; rs < rows * SIDES; rs += few ? SUM_Y * SUM_WARPS : SUM_Y) {
        const int r = rs / SIDES, side = rs % SIDES;
        const int a = few ? 0 : parts * warp / SUM_WARPS, b = few ? parts : parts * (warp + 1) / SUM_WARPS;
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 8
        for (int k = a; k < b; ++k) {
            const float* src = (KV ? w.kv_part : w.q_part) + (((2LL * (first + k) + (k == 0)) * cap + r) * SIDES + side) * DP;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += src[lane + 32 * e];
        }
        if (!few) {
#pragma unroll
            for (int e = 0; e < E; ++e) sh[warp][lane + 32 * e] = o[e];
            __syncthreads();
            if (warp == 0)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    o[e] = sh[0][lane + 32 * e];
                    for (int k = 1; k < SUM_WARPS; ++k) o[e] += sh[k][lane + 32 * e];
                }
            __syncthreads();
        }
        if (few || warp == 0) {
            const int n = it.t * BWD_ROWS + r;
            long long out_row;
            bool masked;
            int keys = g.nk;
            if (KV) {
                out_row = (long long)(g.k0 + n) * p.kv_heads + it.h;
                masked = key_place(p, g, it.s, n).at < 0;
            } else {
                const PackedRow pr = packed_row(p, g, it.h, n);
                keys = keys_of_row(p, g, pr.row - g.q0);
                out_row = (long long)pr.row * p.heads + pr.head;
                masked = w.stats[out_row].x == INFINITY;
            }
            masked = masked || (side == 0 && reads_one_key(p, g, keys));
            const float finish = KV && side ? (F16 ? 0x1p-14f : 1.f) : p.scale / factor;
            T* out = (T*)(KV ? (side ? p.gv : p.gk) : p.gq);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (out && lane + 32 * e < p.D) out[out_row * p.D + lane + 32 * e] = Half<T>::from(masked ? 0.f : o[e] * finish);
        }
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(SUM_WARPS * 32) attention_sum_kernel(const AttnParams p, const BwdWork w, const int kv_blocks) {
    wait_for_previous_kernel();
    if ((int)blockIdx.x < kv_blocks) sum_pass<T, DP, true>(p, w, blockIdx.x);
    else sum_pass<T, DP, false>(p, w, (int)blockIdx.x - kv_blocks);
}

// clears the norms (fp16); counts the units of every segment where the blocks do not
static __global__ void __launch_bounds__(PLAN_THREADS) backward_plan_kernel(const AttnParams p, const BwdWork w, const bool norms) {
    let_next_kernel_start();
    if (norms) for (int i = blockIdx.x * PLAN_THREADS + threadIdx.x; i < 2 * p.n_seg; i += 2 * PLAN_THREADS) w.norms[i] = 0;
    long long* units = blockIdx.x == 0 ? w.kv_start_unit : w.q_start_unit;
    if (!units) return;
    if (p.causal) { if (blockIdx.x == 0) plan_units<BwdCut<true, true>>(p, units); else plan_units<BwdCut<false, true>>(p, units); }
    else if (blockIdx.x == 0) plan_units<BwdCut<true, false>>(p, units);
    else plan_units<BwdCut<false, false>>(p, units);
}

static size_t backward_carve(const AttnParams& p, void* ws, BwdWork* w) {
    const size_t slots = 2 * (size_t)MAX_SMS, dp = p.D > 64 ? 128 : 64;
    const long long packed = (long long)p.n_q * p.group;
    w->kv_rows = p.n_kv < BWD_ROWS ? p.n_kv : BWD_ROWS;
    w->q_rows = (int)(packed < BWD_ROWS ? packed : BWD_ROWS);
    Carver cv(ws);
    const bool counted_there = counts_itself(p, BWD_ROWS, p.item_cost != 0);
    w->kv_start_unit = counted_there ? nullptr : cv.take<long long>((size_t)p.n_seg + 1);
    w->q_start_unit = counted_there ? nullptr : cv.take<long long>((size_t)p.n_seg + 1);
    w->kv_joints = cv.take<Joint>(MAX_SMS);
    w->q_joints = cv.take<Joint>(MAX_SMS);
    w->norms = cv.take<uint32_t>(2 * (size_t)p.n_seg);
    w->stats = cv.take<float2>((size_t)p.n_q * p.heads);
    w->kv_part = cv.take<float>(slots * w->kv_rows * 2 * dp);
    w->q_part = cv.take<float>(slots * w->q_rows * dp);
    return cv.off;
}
size_t attention_backward_bytes(const AttnParams& p) { BwdWork w; return backward_carve(p, nullptr, &w); }

template <typename T, int DP>
static tiga_status launch_backward(AttnParams p, const BwdWork& w, cudaStream_t s) {
    TileMaps maps;
    make_tile_maps(&p, operand_type<T>() == 1, &maps);
    const int sms = attention_grid();
    if (sms <= 0) return TIGA_ERR_CUDA;
    const int kv_blocks = (p.gk || p.gv) && p.n_kv ? sms : 0, q_blocks = p.gq && p.n_q ? sms : 0;
    if (kv_blocks + q_blocks == 0) return TIGA_OK;
    const auto kernel = p.causal ? attention_backward_kernel<T, DP, true> : attention_backward_kernel<T, DP, false>;
    TIGA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Bwd<DP>::SMEM));
    // a row of values costs about half of one of queries
    const long long q_work = (long long)p.n_q * p.heads, v_work = operand_type<T>() == 0 ? ((long long)p.n_kv * p.kv_heads + 1) / 2 : 0;
    const long long grid = prepare_blocks(p, q_work + v_work, DP / 8, sms);
    const int prep_v = !v_work ? 0 : grid == 1 ? 1 : (int)min(max(grid * v_work / (q_work + v_work), 1LL), grid - 1);
    const int prep_q = grid == 1 ? 1 : (int)grid - prep_v;
    const bool plan = w.kv_start_unit || (operand_type<T>() == 0 && grid > 1);
    if (plan) {
        backward_plan_kernel<<<counted(2), PLAN_THREADS, 0, s>>>(p, w, operand_type<T>() == 0);
        TIGA_CUDA_TRY(launch_after(attention_prepare_kernel<T, DP / 8>, dim3((unsigned)grid), PREP_THREADS, 0, s, p, w, prep_q, prep_v));
    } else attention_prepare_kernel<T, DP / 8><<<counted((unsigned)grid), PREP_THREADS, 0, s>>>(p, w, prep_q, prep_v);
    TIGA_CUDA_TRY(launch_after(kernel, dim3(kv_blocks + q_blocks), BWD_THREADS, Bwd<DP>::SMEM, s, p, w, maps, kv_blocks));
    // tiles of a single step are whole
    if ((kv_blocks && (long long)p.n_q * p.group > BWD_STEP) || (q_blocks && p.n_kv > BWD_STEP)) TIGA_CUDA_TRY(launch_after(attention_sum_kernel<T, DP>, dim3(kv_blocks + q_blocks, SUM_Y), SUM_WARPS * 32, 0, s, p, w, kv_blocks));
    return launch_status();
}

tiga_status attention_backward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s) {
    BwdWork w;
    backward_carve(p, on_sectors(ws), &w);
    if (bf16) return p.D > 64 ? launch_backward<__nv_bfloat16, 128>(p, w, s) : launch_backward<__nv_bfloat16, 64>(p, w, s);
    return p.D > 64 ? launch_backward<__half, 128>(p, w, s) : launch_backward<__half, 64>(p, w, s);
}

}  // namespace tiga
