// Online-softmax reducer over dense and paged relations, forward, on the fifth-generation tensor cores.
#include "attention_shared.cuh"
#include "attention_tiles.cuh"

namespace tiga {

// A block holds a tile of 256 packed rows as two halves of 128, two warpgroups of softmax threads for each (a row has two threads,
// for 64 of a step's columns each), and goes through the keys in steps of 128:
//   producers (4 warps)   bring query and key / value rows to shared memory (attention_tiles.cuh), zeros for what is masked, missing
//                         or behind the head's width; a ring of key and value tiles in the order K0 V0 K1 V1 ...
//   one thread            issues S = Q K^T (to tensor memory) and O += P V (P from tensor memory, O stays there for the whole tile)
//   softmax warpgroups    running maximum, P = exp2(S - m) in 16 bits over S's own columns, running mass
// While one half's softmax runs, the tensor cores work for the other.  A tile of at most 128 rows has one half; then the warpgroups
// of the halves take the even and the odd steps with a state each, joined at the end, so a single token keeps both busy too.
// The accumulator is rescaled only when a row's maximum grew by more than 2^8 since the last time: weights up to 2^8 do no harm,
// and the mass carries the same factor.
// What bounds it: the chain S -> maximum -> P -> O of a half, 3700 cycles a step of 128 keys at a width of 128 (3550 at 64; what twice the keys
// take more) where its products take 1024 and its 16384 exponentials another 1024.  Two threads a row halve what one would take (a warp alone on its scheduler needs
// about 13 cycles a column); the exchange of their maxima costs 100.  4 segments of 4096 rows and keys, 16/4 heads of 128, bf16: 543 us
// alone, 1.0 PFLOP/s; single tokens read their cache at 6.3 TB/s between the ends of items.
constexpr int FWD_SOFTMAX_WARPS = 16, FWD_PRODUCER = FWD_SOFTMAX_WARPS, FWD_MMA = FWD_PRODUCER + 4, FWD_WALKER = FWD_MMA + 1;
constexpr int FWD_THREADS = 32 * (FWD_WALKER + 1), FWD_ROWS = 256, FWD_STEP = 128;
template <int MODE> using FwdCut = Cut<FWD_ROWS, FWD_STEP, false, MODE>;
typedef FwdCut<CUT_LINE> SharedCut;
constexpr int MASK_RING = 8;            // the producers are at most 6 steps ahead of the softmax (ring of at most 10 tiles)
constexpr float RESCALE_AT = 8.f;

template <int DP> struct Fwd {
    static constexpr int TILE = 128 * DP * 2;
    static constexpr int SLOTS = DP == 128 ? 5 : 10;
    static constexpr int CONTROL = 2 * TILE + SLOTS * TILE;
    static constexpr int SMEM = CONTROL + 3 * 1024;
};

struct FwdControl {
    unsigned long long full[10], empty[10], q_full, q_empty, s_full[2], p_full[2], o_full[2], mask_full[MASK_RING], drain;
    ItemRing items;
    alignas(8) unsigned char walk[sizeof(Walker<FwdCut<CUT_COSTS>>)];      // a Walker of the kernel's cut
    uint32_t tmem, abort_word, mask[MASK_RING][4];
    float share[2][2][128];             // what a row's threads tell each other
};
static_assert(sizeof(FwdControl) <= 3 * 1024, "control block");

struct FwdWork {
    long long* unit_start;          // NULL: the blocks count for themselves
    float2* part_ml;                // [2 * grid][rows]: reference of the exponents (log2), mass
    float* part_o;                  // [2 * grid][rows][DP]: unnormalised
    Joint* joints;                  // [grid]
    int rows;                       // packed rows that a partial state holds at most
    // shared prefixes
    int n_groups, n_seq;
    long long state_rows;           // rows that there is room for
    const int32_t* line_row;        // [n_groups + n_seq]: the row of the page table that a segment of the line reads
    const long long* line_state;    // [n_groups + n_seq]: what is added to a row's number for its place among the states
    const int32_t* first_member;    // [n_groups]
    const Walker<SharedCut>* walks; // [grid]: where the blocks' pieces of the line begin
    const long long* state_start;   // [n_groups + 1]: rows of the groups in front that share
    float2* state_ml;               // [2][state_rows][heads]: as part_ml, of the shared and of the own keys
    float* state_o;                 // [2][state_rows][heads][DP]
};
// Whether a segment of the line has the only state of its rows.
__device__ __forceinline__ bool only_state(const FwdWork& w, int s, int k0) { return s >= w.n_groups && k0 == 0; }

static __global__ void __launch_bounds__(PLAN_THREADS) forward_plan_kernel(const AttnParams p, long long* unit_start) {
    if (p.item_cost) plan_units<FwdCut<CUT_COSTS>>(p, unit_start);
    else plan_units<FwdCut<CUT_STEPS>>(p, unit_start);
}

template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(FWD_THREADS, 1) attention_forward_kernel(const __grid_constant__ AttnParams p, const FwdWork w, const __grid_constant__ TileMaps maps) {
    typedef Fwd<DP> C;
    typedef Walker<FwdCut<MODE>> Walk;
    constexpr bool SHARED = MODE == CUT_LINE;
    extern __shared__ __align__(1024) unsigned char smem[];
    FwdControl& ctl = *reinterpret_cast<FwdControl*>(smem + C::CONTROL);
    const uint32_t q_tile = smem_u32(smem), ring = q_tile + 2 * C::TILE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile uint32_t* abort_word = &ctl.abort_word;
    auto bar = [&](unsigned long long& b) { return smem_u32(&b); };

    wait_for_previous_kernel();
    let_next_kernel_start();
    if (threadIdx.x == 0) {
        items_init(ctl.items, FWD_WALKER);
        for (int i = 0; i < C::SLOTS; ++i) { mbar_init(bar(ctl.full[i]), 128); mbar_init(bar(ctl.empty[i]), 1); }
        mbar_init(bar(ctl.q_full), 256);
        mbar_init(bar(ctl.q_empty), 1);
        for (int x = 0; x < 2; ++x) { mbar_init(bar(ctl.s_full[x]), 1); mbar_init(bar(ctl.p_full[x]), 256); mbar_init(bar(ctl.o_full[x]), 1); }
        for (int i = 0; i < MASK_RING; ++i) mbar_init(bar(ctl.mask_full[i]), 4);
        mbar_init(bar(ctl.drain), 1);
        ctl.abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    Walk walk;
    if (MODE == CUT_COSTS) { if (warp == FWD_WALKER) walk_begin(reinterpret_cast<Walk*>(ctl.walk), p, w.unit_start, blockIdx.x, gridDim.x); }
    else if (MODE == CUT_STEPS) {
        walk.here = false;
        if (warp == FWD_WALKER) walk.here = walk.begin(p, w.unit_start, blockIdx.x, gridDim.x);
    }
    if (warp == FWD_MMA) tmem_alloc(smem_u32(&ctl.tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = ctl.tmem;
    // tensor memory: S of half x at 128 x, O at 256 + DP x

    if (warp == FWD_WALKER) {
        if (lane == 0) {
            if (MODE == CUT_COSTS) walk = *reinterpret_cast<Walk*>(ctl.walk);
            if constexpr (SHARED) walk = w.walks[blockIdx.x];
            w.joints[blockIdx.x] = joint_of(p, walk, walk.here && (!SHARED || only_state(w, walk.s, walk.g.k0)), blockIdx.x);
            items_hand_out(ctl.items, p, walk, walk.here);
        }
        __syncwarp();
    } else if (warp >= FWD_PRODUCER && warp < FWD_MMA) {
        // ---------------------------------------------------------------- producers
        const int pw = warp - FWD_PRODUCER;
        uint32_t tiles = 0, steps = 0, items = 0;
        bool ok = true;
        auto wait = [&](unsigned long long& b, uint32_t parity) { return ok = __all_sync(~0u, mbar_wait(bar(b), parity & 1, abort_word)); };
        auto slot_free = [&]() { return tiles < (uint32_t)C::SLOTS || wait(ctl.empty[tiles % C::SLOTS], tiles / C::SLOTS + 1); };
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const Segment g = e.segment();
            const int i0 = e.i0, i1 = e.i1, h = e.h, row = SHARED ? w.line_row[e.s] : e.s;
            auto place = [&](int i) {
                const int j = i * FWD_STEP + 32 * pw + lane;
                return j >= g.nk ? Place{-1, 0} : SHARED ? shared_place(p, g, row, j) : key_place(p, g, row, j);
            };
            Place at = place(i0);
            for (int i = i0; i < i1 && ok; ++i, ++steps) {
                const Place here = at;
                const uint32_t valid = __ballot_sync(~0u, here.at >= 0);
                if (lane == 0) {
                    ctl.mask[steps % MASK_RING][pw] = valid;
                    mbar_arrive(bar(ctl.mask_full[steps % MASK_RING]));
                }
                if (i + 1 < i1) at = place(i + 1);
                for (int kv = 0; kv < 2; ++kv, ++tiles) {
                    if (!slot_free()) break;
                    fetch_keys<DP>(ring + (tiles % C::SLOTS) * C::TILE, 32 * pw, bar(ctl.full[tiles % C::SLOTS]), p, maps, kv, here, h, p.q);
                }
                if (i == i0 && ok) {            // the queries' tile may still be in use by the item before: its first keys are on their way
                    if (items && !wait(ctl.q_empty, items - 1)) break;
                    const int rows = min(g.nq * p.group - e.t * FWD_ROWS, FWD_ROWS);
                    for (int x = 0; x < 2; ++x) {
                        const int r = x * 128 + 32 * pw + lane;
                        if (x == 1 && rows <= 128) {
                            if (lane == 0) mbar_arrive(bar(ctl.q_full), 32);
                        } else fetch_packed<DP>(q_tile + x * C::TILE, 32 * pw, bar(ctl.q_full), p, g, maps, false, h, e.t * FWD_ROWS + r, r < rows, p.q);
                    }
                    ++items;
                }
            }
            item_return(ctl.items, item);
        }
        cp_async_wait_all();
        if (*abort_word) {          // boxes may still be on their way: their tiles, as far as they were asked for
            for (uint32_t k = tiles < (uint32_t)C::SLOTS ? 0 : tiles - C::SLOTS; k < tiles; ++k) mbar_wait_for(bar(ctl.full[k % C::SLOTS]), (k / C::SLOTS) & 1, HALF_A_SECOND);
            if (items) mbar_wait_for(bar(ctl.q_full), (items - 1) & 1, HALF_A_SECOND);
        }
    } else if (warp == FWD_MMA) {
        // ---------------------------------------------------------------- matrix instructions
        // the warp goes its way together, one thread issues
        const uint32_t s_shape = mma_shape<T>(128, false) | (p.scale < 0.f ? MMA_NEGATE_A : 0), o_shape = mma_shape<T>(DP, true);
        uint32_t tile0 = 0, items = 0, done0 = 0, done1 = 0;     // done: p_full phases consumed
        bool ok = true;
        // descriptors differ in their address alone: a product costs its instruction and an addition (built anew each time, about
        // 100 cycles of this one thread, they bounded the kernel)
        const uint32_t q_desc = smem_desc(q_tile, 16), k_desc = smem_desc(ring, 16), v_desc = smem_desc(ring, 128 * 128);
        auto slot = [&](uint32_t tile) { return (tile % C::SLOTS) * (uint32_t)(C::TILE / 16); };
        auto wait = [&](unsigned long long& b, uint32_t parity) { ok = __all_sync(~0u, ok && mbar_wait(bar(b), parity & 1, abort_word)); };
        auto wait_tile = [&](uint32_t tile) {
            wait(ctl.full[tile % C::SLOTS], tile / C::SLOTS);
            fence_async_proxy();
        };
        auto release = [&](uint32_t tile) { if (elected()) mma_commit(bar(ctl.empty[tile % C::SLOTS])); };
        auto scores = [&](int x, int half, uint32_t tile) {
            const uint32_t q = q_desc + half * (C::TILE / 16), k = k_desc + slot(tile);
            if (elected()) {
#pragma unroll
                for (int c = 0; c < DP / 16; ++c)
                    if (c * 16 < p.D) mma_ss(tmem + 128 * x, q + piece(c), k + piece(c), s_shape, c > 0);
                mma_commit(bar(ctl.s_full[x]));
            }
            __syncwarp();
        };
        auto values = [&](int x, uint32_t tile, bool add) {
            wait(ctl.p_full[x], x ? done1++ : done0++);
            if (!ok) return;
            tmem_fence_after();
            const uint32_t v = v_desc + slot(tile);
            const uint32_t o = tmem + 256 + DP * x, a = tmem + 128 * x;
            if (elected()) {
                mma_ts(o, a, v, o_shape, add);
#pragma unroll
                for (int k = 1; k < 8; ++k) mma_ts(o, a + (k / 2) * 32 + (k % 2) * 8, v + k * (2048 / 16), o_shape, true);
                mma_commit(bar(ctl.o_full[x]));
            }
            __syncwarp();
        };
        for (;; ++items) {
            const Item& e = item_take(ctl.items, items);
            if (e.steps == 0) break;
            const int n = e.i1 - e.i0;
            const bool two = e.nq * p.group - e.t * FWD_ROWS > 128;
            item_return(ctl.items, items);
            if (!ok) continue;
            const int ahead = two ? 1 : 2;              // steps between two of a half
            wait(ctl.q_full, items);
            // i: the step whose values are next; its half's (two: both halves') next scores follow
            for (int i = -ahead; i < n && ok; ++i) {
                const uint32_t v = tile0 + 2 * i + 1, k_next = tile0 + 2 * (i + ahead);
                const bool more_keys = i + ahead < n;
                const int x = two ? 0 : i & 1;
                if (i >= 0) {
                    wait_tile(v);
                    values(x, v, i >= ahead);
                    if (!two && ok) release(v);
                }
                if (more_keys) wait_tile(k_next);
                if (!ok) break;
                if (more_keys) scores(x, 0, k_next);
                if (two && i >= 0) {
                    values(1, v, i > 0);
                    if (!ok) break;
                    release(v);
                }
                if (two && more_keys) scores(1, 1, k_next);
                if (more_keys) release(k_next);
                if (i + ahead == n - 1 && elected()) mma_commit(bar(ctl.q_empty));      // the last scores: the next item's queries may come
            }
            tile0 += 2 * n;
        }
        if (elected()) mma_commit(bar(ctl.drain));
        mbar_wait_for(bar(ctl.drain), 0, HALF_A_SECOND);
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax
        const int x = warp / 8, y = warp / 4 % 2;           // half, and which of its columns
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const int row = threadIdx.x & 127;
        const uint32_t S = tmem + 128 * x + lanes + 64 * y, O = tmem + 256 + lanes;
        const float scale2 = fmaxf(fabsf(p.scale) * LOG2E_F, 1e-30f);       // (not zero: masked scores are -inf)
        constexpr float BIAS = operand_type<T>() == 0 ? 7.f : 0.f;          // fp16: weights up to 2^15, so that small ones keep their digits
        // The threads of a half, and all of them, meet here; everyone comes the same number of times, after a failed wait too.
        auto meet_half = [&]() { if (x) asm volatile("bar.sync 2, 256;" ::: "memory"); else asm volatile("bar.sync 1, 256;" ::: "memory"); };
        auto meet_all = [&]() { asm volatile("bar.sync 3, 512;" ::: "memory"); };
        uint32_t step0 = 0, s_done = 0, o_done0 = 0, o_done1 = 0;       // steps, scores of this half, values of each half in the items before
        bool ok = true;
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const int n = e.i1 - e.i0;
            const int rows = min(e.nq * p.group - e.t * FWD_ROWS, FWD_ROWS);
            const bool two = rows > 128;
            const int tile_row = two ? x * 128 + row : row;
            const bool valid = tile_row < rows;
            const bool warp_on = (tile_row & ~31) < rows;
            const int limit = (p.causal && valid ? keys_of_row(p, e.segment(), (e.t * FWD_ROWS + tile_row) / p.group) : e.nk) - e.i0 * FWD_STEP - 64 * y;
            const uint32_t o_mine = x ? o_done1 : o_done0;
            float m = -INFINITY, l = 0.f;               // reference of the exponents (log2), this thread's mass relative to 2^(m - BIAS)
            uint32_t mine = 0;                          // steps of this half's threads in this item
            for (int i = two ? 0 : x; i < n; i += two ? 1 : 2, ++mine, ++s_done) {
                const uint32_t step = step0 + i, ring_at = step % MASK_RING;
                ok = ok && mbar_wait(bar(ctl.mask_full[ring_at]), (step / MASK_RING) & 1, abort_word) && mbar_wait(bar(ctl.s_full[x]), s_done & 1, abort_word);
                ok = __all_sync(~0u, ok);
                tmem_fence_after();
                const bool work = ok && warp_on;
                uint32_t v[32], keep[2];            // 32 of the 64 columns are held, the others read twice: registers
                bool whole = true;
                float top = -INFINITY;
                auto hide = [&](uint32_t kept) {
                    if (!whole)
#pragma unroll
                        for (int k = 0; k < 32; ++k) if (!(kept >> k & 1)) v[k] = 0xff800000u;
                };
                if (work) {
                    tmem_ld32(S, v);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int bits = limit - i * FWD_STEP - 32 * c;
                        keep[c] = ctl.mask[ring_at][2 * y + c] & (bits >= 32 ? ~0u : bits <= 0 ? 0u : (1u << bits) - 1);
                    }
                    whole = __all_sync(~0u, (keep[0] & keep[1]) == ~0u);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (c) tmem_ld32(S + 32, v);
                        tmem_wait_ld(v);
                        hide(keep[c]);
                        float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            t0 = max3(t0, __uint_as_float(v[k]), __uint_as_float(v[k + 1]));
                            t1 = max3(t1, __uint_as_float(v[k + 2]), __uint_as_float(v[k + 3]));
                        }
                        top = max3(top, t0, t1);
                    }
                }
                ctl.share[x][y][row] = top;
                meet_half();
                if (work) {
                    top = fmaxf(top, ctl.share[x][1 - y][row]) * scale2;
                    const bool grown = top > m + RESCALE_AT || (m == -INFINITY && top > -INFINITY);
                    if (__any_sync(~0u, grown)) {
                        const float m_new = grown ? top : m;
                        const float fade = grown ? ex2(m - m_new) : 1.f;
                        if (mine) {
                            ok = mbar_wait(bar(ctl.o_full[x]), (o_mine + mine - 1) & 1, abort_word);
                            ok = __all_sync(~0u, ok);
                            tmem_fence_after();
                            if (ok)
#pragma unroll 1
                                for (int c = 0; c < DP / 16; ++c) {         // this thread's half of the features, eight at a time
                                    const uint32_t at = O + DP * x + y * (DP / 2) + 8 * c;
                                    uint32_t o[8];
                                    tmem_ld8(at, o);
                                    tmem_wait_ld(o);
#pragma unroll
                                    for (int k = 0; k < 8; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * fade);
                                    tmem_st8(at, o);
                                }
                        }
                        m = m_new;
                        l *= fade;
                    }
                    const float shift = m == -INFINITY ? 0.f : BIAS - m;
                    const f32x2 sc2 = dup2(scale2), sh2 = dup2(shift);
                    f32x2 sum = pack2(0.f, 0.f);
#pragma unroll
                    for (int c = 1; c >= 0; --c) {
                        if (c == 0) {
                            tmem_ld32(S, v);
                            tmem_wait_ld(v);
                            hide(keep[0]);
                        }
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float a, b;
                            unpack2(fma2(pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), sc2, sh2), a, b);
                            a = ex2(a);
                            b = ex2(b);
                            sum = add2(sum, pack2(a, b));
                            v[k] = pack_half<T>(a, b);
                        }
                        tmem_st16(S + 32 * c, v);           // in the first half of their own columns
                    }
                    float a, b;
                    unpack2(sum, a, b);
                    l += a + b;
                    tmem_wait_st();
                }
                tmem_fence_before();
                mbar_arrive(bar(ctl.p_full[x]));
            }
            // ---- the item's end: the row's mass; a short tile's two states are joined; then the rows are finished or put aside
            const uint32_t made0 = two ? n : (n + 1) / 2, made1 = two ? n : n / 2;
            // Each half waits for its own products alone: the scores of its last step came behind the products of the step before, so the
            // phase that it waits for is the one under way.  (The other half's may lag by more than a phase, which a parity cannot tell.)
            const uint32_t made = x ? made1 : made0;
            if (ok && made) ok = mbar_wait(bar(ctl.o_full[x]), (o_mine + made - 1) & 1, abort_word);
            ok = __all_sync(~0u, ok);
            if (!ok) l = __int_as_float(0x7fffffff);
            tmem_fence_after();
            ctl.share[x][y][row] = l;
            float w0 = 1.f, w1 = 0.f;               // factors of the accumulators: two halves have one each
            if (two) {
                meet_half();
                l += ctl.share[x][1 - y][row];
            } else {
                tmem_fence_before();
                meet_all();                     // both accumulators are complete, and may be read
                tmem_fence_after();
                const float la = ctl.share[0][0][row] + ctl.share[0][1][row], lb = ctl.share[1][0][row] + ctl.share[1][1][row];
                meet_all();
                if (y == 0) ctl.share[x][0][row] = m;
                meet_all();
                const float ma = ctl.share[0][0][row], mb = ctl.share[1][0][row];
                m = fmaxf(ma, mb);
                w0 = ma == -INFINITY ? 0.f : ex2(ma - m);
                w1 = mb == -INFINITY ? 0.f : ex2(mb - m);
                l = la * w0 + lb * w1;
            }
            const PackedRow pr = packed_row(p, e.segment(), e.h, e.t * FWD_ROWS + tile_row);
            const long long out_row = (long long)pr.row * p.heads + pr.head;
            // a state that is not the rows' only one, or not whole, is put aside
            const bool all_steps = n == e.steps, whole_tile = all_steps && (!SHARED || only_state(w, e.s, e.k0));
            long long part = (2LL * blockIdx.x + (e.i0 == 0)) * w.rows + tile_row;
            float* put_aside = w.part_o;
            float2* put_ml = w.part_ml;
            if (SHARED && all_steps && !whole_tile) {
                part = ((e.s < w.n_groups ? 0 : w.state_rows) + w.line_state[e.s] + pr.row) * p.heads + pr.head;
                put_aside = w.state_o;
                put_ml = w.state_ml;
            }
            const float finish = l > 0.f || l != l ? 1.f / l : 0.f;
            // this thread's half of the row's features, or its quarter of both states, 16 at a time
            const int f0 = two ? y * (DP / 2) : (2 * x + y) * (DP / 4), f1 = f0 + (two ? DP / 2 : DP / 4);
            if (warp_on)
#pragma unroll 1
                for (int f = f0; f < f1; f += 16) {
                    uint32_t v[16], u[16];
                    tmem_ld16(O + (two ? DP * x : 0) + f, v);
                    tmem_ld16(O + DP + f, u);           // (wanted in short tiles with a second state only)
                    tmem_wait_ld(v);
                    tmem_wait_ld(u);
                    if (!two)
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            v[k] = __float_as_uint(__uint_as_float(v[k]) * w0 + (made1 ? __uint_as_float(u[k]) * w1 : 0.f));
                    if (whole_tile) {
                        uint4 o[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t h[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                h[k] = finish == 0.f ? 0u : pack_half<T>(__uint_as_float(v[8 * c + 2 * k]) * finish, __uint_as_float(v[8 * c + 2 * k + 1]) * finish);
                            o[c] = make_uint4(h[0], h[1], h[2], h[3]);
                        }
                        store_pieces(o, (T*)p.out + out_row * p.D + f, valid, (p.D - f) / 8, p.whole_sectors & WHOLE_OUT);
                    } else if (valid) {
                        store_sector(put_aside + part * DP + f, v);
                        store_sector(put_aside + part * DP + f + 8, v + 8);
                    }
                }
            if (valid && y == 0 && (two || x == 0)) {
                if (!whole_tile) put_ml[part] = make_float2(m - BIAS, l);
                else if (p.lse) p.lse[out_row] = l == 0.f ? -INFINITY : (m - BIAS + log2f(l)) * LN2_F;
            }
            tmem_fence_before();
            // what was read here (accumulators of both halves, shared words) is free for the next item
            if (two) meet_half();
            else meet_all();
            step0 += n;
            o_done0 += made0;
            o_done1 += made1;
            item_return(ctl.items, item);
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == FWD_MMA) { tmem_fence_after(); tmem_free(tmem, 512); }
}

// Joins the partial states of a tile that several blocks shared, in the order of its steps.  blockIdx.x: the block in which a tile
// ends that began in an earlier one; its rows are dealt over blockIdx.y.  Up to FEW parts: a warp per row.  More (few rows, a long
// axis): the block's warps share a row's parts.
constexpr int JOIN_WARPS = 8, JOIN_Y = 16, JOIN_FEW = 8;

// one of `slices` parts of a block's rows
template <typename T, int DP>
__device__ __forceinline__ void join_block(const AttnParams& p, const FwdWork& w, const int block, const int slice, const int slices) {
    const Joint& j = w.joints[block];
    const int parts = j.parts;
    if (parts == 0) return;
    const Item it = j.item;
    const int first = j.first, rows = min(it.nq * p.group - it.t * FWD_ROWS, FWD_ROWS);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    constexpr int E = DP / 32;
    __shared__ float sh_m[JOIN_WARPS], sh_l[JOIN_WARPS], sh_o[JOIN_WARPS][DP];
    const bool few = parts <= JOIN_FEW;
    for (int r = few ? slice * JOIN_WARPS + warp : slice; r < rows; r += few ? slices * JOIN_WARPS : slices) {
        const int a = few ? 0 : parts * warp / JOIN_WARPS, b = few ? parts : parts * (warp + 1) / JOIN_WARPS;
        float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
        for (int k0 = a; k0 < b; k0 += 32) {
            const int k = k0 + lane;
            float2 ml = make_float2(-INFINITY, 0.f);
            if (k < b) ml = w.part_ml[(2LL * (first + k) + (k == 0)) * w.rows + r];
            float top = ml.x != ml.x ? INFINITY : ml.x;
#pragma unroll
            for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
            top = fmaxf(top, m);
            const float fade = m == -INFINITY ? 0.f : ex2(m - top);
            const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
            float mass = f * ml.y;
#pragma unroll
            for (int d = 16; d; d >>= 1) mass += __shfl_xor_sync(~0u, mass, d);
            l = l * fade + mass;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] *= fade;
            m = top;
            const int here = min(32, b - k0);
#pragma unroll 8
            for (int n = 0; n < here; ++n) {
                const float fn = __shfl_sync(~0u, f, n);
                const float* src = w.part_o + ((2LL * (first + k0 + n) + (k0 + n == 0)) * w.rows + r) * DP;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] += fn * src[lane + 32 * e];
            }
        }
        if (!few) {
            if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
#pragma unroll
            for (int e = 0; e < E; ++e) sh_o[warp][lane + 32 * e] = o[e];
            __syncthreads();
            if (warp == 0) {
                float top = -INFINITY;
                for (int k = 0; k < JOIN_WARPS; ++k) top = fmaxf(top, sh_m[k]);
                l = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = 0.f;
                for (int k = 0; k < JOIN_WARPS; ++k) {
                    const float f = sh_m[k] == -INFINITY ? 0.f : ex2(sh_m[k] - top);
                    l += f * sh_l[k];
#pragma unroll
                    for (int e = 0; e < E; ++e) o[e] += f * sh_o[k][lane + 32 * e];
                }
                m = top;
            }
            __syncthreads();
        }
        if (few || warp == 0) {
            const PackedRow pr = packed_row(p, it.segment(), it.h, it.t * FWD_ROWS + r);
            const long long out_row = (long long)pr.row * p.heads + pr.head;
            const float finish = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (lane + 32 * e < p.D) ((T*)p.out)[out_row * p.D + lane + 32 * e] = Half<T>::from(finish == 0.f ? 0.f : o[e] * finish);
            if (lane == 0 && p.lse) p.lse[out_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2_F;
        }
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(JOIN_WARPS * 32) attention_join_kernel(const AttnParams p, const FwdWork w) {
    wait_for_previous_kernel();
    join_block<T, DP>(p, w, blockIdx.x, blockIdx.y, JOIN_Y);
}

size_t attention_forward_carve(const AttnParams& p, void* ws, FwdWork* w) {
    const size_t slots = 2 * (size_t)MAX_SMS;
    const long long packed = (long long)p.n_q * p.group;
    w->rows = (int)(packed < FWD_ROWS ? packed : FWD_ROWS);
    Carver cv(ws);
    w->unit_start = cv.take<long long>((size_t)p.n_seg + 1);       // (room for it whether or not this call needs it)
    if (counts_itself(p, FWD_ROWS, p.item_cost != 0)) w->unit_start = nullptr;
    w->joints = cv.take<Joint>(MAX_SMS);
    w->part_ml = cv.take<float2>(slots * w->rows);
    w->part_o = cv.take<float>(slots * w->rows * (p.D > 64 ? 128 : 64));
    return cv.off;
}
size_t attention_forward_bytes(const AttnParams& p) { FwdWork w; return attention_forward_carve(p, nullptr, &w); }

template <typename T, int DP>
static tiga_status launch_forward(AttnParams p, const FwdWork& w, cudaStream_t s) {
    TileMaps maps;
    make_tile_maps(&p, operand_type<T>() == 1, &maps);
    const int sms = attention_grid();
    if (sms <= 0) return TIGA_ERR_CUDA;
    // asked for on every call: the attribute belongs to the current device
    const auto kernel = p.item_cost ? attention_forward_kernel<T, DP, CUT_COSTS> : attention_forward_kernel<T, DP, CUT_STEPS>;
    TIGA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Fwd<DP>::SMEM));
    if (w.unit_start) forward_plan_kernel<<<counted(1), PLAN_THREADS, 0, s>>>(p, w.unit_start);
    if (w.unit_start) TIGA_CUDA_TRY(launch_after(kernel, dim3(sms), FWD_THREADS, Fwd<DP>::SMEM, s, p, w, maps));
    else kernel<<<counted((unsigned)sms), FWD_THREADS, Fwd<DP>::SMEM, s>>>(p, w, maps);
    // tiles of a single step are whole
    if (p.table || p.n_kv > FWD_STEP) TIGA_CUDA_TRY(launch_after(attention_join_kernel<T, DP>, dim3(sms, JOIN_Y), JOIN_WARPS * 32, 0, s, p, w));
    return launch_status();
}

tiga_status attention_forward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s) {
    FwdWork w;
    attention_forward_carve(p, on_sectors(ws), &w);
    if (bf16) return p.D > 64 ? launch_forward<__nv_bfloat16, 128>(p, w, s) : launch_forward<__nv_bfloat16, 64>(p, w, s);
    return p.D > 64 ? launch_forward<__half, 128>(p, w, s) : launch_forward<__half, 64>(p, w, s);
}

// ------------------------------------------------------------------------------------------------ shared prefixes

// Sequences of a group read their first P positions from the same pages.  Taken one by one, a new token's few rows fill little of a tile,
// and every sequence reads the shared pages again.  So a group's rows, which lie one behind the other, are one segment over the shared
// positions (a dense block: each of them reads all), and every sequence's rows another over the positions behind them; both kinds stand
// in one line, shared ones first, and are cut as everything else.  A row then has two states (maximum, mass, accumulator), which a last
// kernel joins.  The shared positions are a hint, not a part of the result: they are cut so that every row of the group reads all of
// them, and a group shares nothing where that would not make fewer steps.
//
// What the group's sequences cost alone, in halves of a step for every 128 shared positions, against the group together.
__device__ __forceinline__ int tile_halves(int packed) {            // of a segment's tiles; one of at most 128 rows costs half of a full one
    const int rest = packed % FWD_ROWS;
    return 2 * (packed / FWD_ROWS) + (rest == 0 ? 0 : rest <= 128 ? 1 : 2);
}
// Whether a group shares: halves of a step that it saves, more than 8 for each of its tiles (one new token each, 32/8 heads of 128, on the device,
// shared and alone: 8 users of 4096 positions 33 and 43 us, 16 groups of 8 of 256 positions 72 and 78, 4 users of 128 positions 26.6 and
// 22.7.  It is off where states outweigh steps, 64 users of 128 positions 51 and 43, and where steps are many but users two, 32 pairs of 1024
// positions 74 and 83.)
constexpr int SHARED_PAYS = 8;
// What a tile costs beside its steps, of which each is two or three units (attention_shared.cuh).  64 users of 8192 positions and 48 samples of 16384
// (32/8 heads; width 128, then 64): 84 and 118, 75 and 105 us; with a cost of 1 89 and 187, 76 and 147; of 10 99 and 124, 87 and 113; with
// equal steps 101 and 132, 88 and 110.
constexpr int SHARED_ITEM_COST = 5;
// Rows of a group that shares: up to a full tile for each member on average (longer chunks fill their tiles alone).
__host__ __device__ __forceinline__ long long most_state_rows(long long n_seq, long long n_q, int group) {
    const long long n = (n_seq * FWD_ROWS + group - 1) / group;
    return n < n_q ? n : n_q;
}

struct SharedPlan {
    Segment* line;
    int32_t *line_row, *first_member;
    long long *line_state, *state_start, *unit_start;
    Walker<SharedCut>* walks;
};

// One block: a warp for each group, a thread for each sequence, then the units.  What is looked up again and again lies in shared memory where
// it fits: this kernel is a chain of latencies in front of everything else.
constexpr int PLAN_HELD = 768;
static __global__ void __launch_bounds__(PLAN_THREADS) shared_plan_kernel(AttnParams p, Prefixes x, const SharedPlan plan, const long long state_rows, const int sms) {
    __shared__ int32_t rows[PLAN_HELD], lengths[PLAN_HELD], members[PLAN_HELD], said[PLAN_HELD];
    __shared__ Segment held[PLAN_HELD];             // of the groups, and what is added to their rows' numbers
    __shared__ long long held_state[PLAN_HELD], held_units[PLAN_HELD];
    __shared__ long long totals[PLAN_THREADS / 32];
    wait_for_previous_kernel();
    let_next_kernel_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, n_seq = p.n_seg;
    if (n_seq < PLAN_HELD) {
        if ((int)threadIdx.x <= n_seq) rows[threadIdx.x] = p.q_start[threadIdx.x];
        if ((int)threadIdx.x < n_seq) lengths[threadIdx.x] = p.kv_len[threadIdx.x];
        p.q_start = rows;
        p.kv_len = lengths;
    }
    const bool few = x.n_groups < PLAN_HELD;
    if (few) {
        if ((int)threadIdx.x <= x.n_groups) members[threadIdx.x] = x.group_start[threadIdx.x];
        if ((int)threadIdx.x < x.n_groups) said[threadIdx.x] = x.shared[threadIdx.x];
        x.group_start = members;
        x.shared = said;
    }
    Segment* groups = few ? held : plan.line;
    long long* states = few ? held_state : plan.line_state;
    __syncthreads();
    const long long most = min(min(p.max_pages * p.page_size, MOST_ROWS), 1LL << 30);
    for (int g = warp; g < x.n_groups; g += PLAN_THREADS / 32) {
        const int a = clamp_to(x.group_start[g], n_seq), b = max(clamp_to(x.group_start[g + 1], n_seq), a);
        int shared = (int)min((long long)max(x.shared[g], 0), most), halves = 0, reader = n_seq;
        for (int s = a + lane; s < b; s += 32) {
            const Segment e = segment_of(p, s);
            if (e.nq == 0) continue;            // (reads nothing: its length and its pages may be another's by now)
            reader = min(reader, s);
            shared = min(shared, p.causal ? max(e.length - e.nq + 1, 0) : e.length);
            halves += tile_halves(e.nq * p.group);
        }
        shared = __reduce_min_sync(~0u, shared);
        halves = __reduce_add_sync(~0u, halves);
        reader = __reduce_min_sync(~0u, reader);
        const int q0 = clamp_to(p.q_start[a], p.n_q), nq = max(clamp_to(p.q_start[b], p.n_q) - q0, 0);
        const long long steps = quotient(shared + FWD_STEP - 1, FWD_STEP), tiles = quotient((long long)nq * p.group + FWD_ROWS - 1, FWD_ROWS);
        const bool pays = (long long)nq * p.group <= (long long)(b - a) * FWD_ROWS && (halves - tile_halves(nq * p.group)) * steps > SHARED_PAYS * tiles && nq < 1 << 30;
        if (lane == 0) {
            groups[g] = {q0, pays ? nq : 0, 0, pays ? shared : 0, pays ? shared + nq : 0};
            plan.line_row[g] = reader;          // (n_seq: the group has no rows, and nothing is looked up)
        }
    }
    __syncthreads();
    if (warp == 0) {            // places of the groups' states; a group for which there is no room (bounds that overlap) shares nothing
        long long base = 0;
        for (int g0 = 0; g0 < x.n_groups; g0 += 32) {
            const int g = g0 + lane;
            const long long n = g < x.n_groups ? groups[g].nq : 0, run = warp_running(n);
            if (g < x.n_groups) {
                plan.state_start[g] = base + run - n;
                states[g] = base + run - n - groups[g].q0;
                if (base + run > state_rows) groups[g] = {0, 0, 0, 0, 0};
                plan.first_member[g] = clamp_to(x.group_start[g], n_seq);
            }
            base += __shfl_sync(~0u, run, 31);
        }
        if (lane == 0) plan.state_start[x.n_groups] = min(base, state_rows);
    }
    __syncthreads();
    // the line, and its units
    const int n_line = x.n_groups + n_seq;
    long long* units = n_line < PLAN_HELD ? held_units : plan.unit_start;
    long long before = 0;
    for (int i0 = 0; i0 < n_line; i0 += PLAN_THREADS) {
        const int i = i0 + (int)threadIdx.x, s = i - x.n_groups;
        long long n = 0;
        if (i < n_line) {
            Segment e;
            long long state = 0;
            if (s < 0) {
                e = groups[i];
                state = states[i];
            } else {
                e = segment_of(p, s);
                int lo = 0, hi = x.n_groups;                // the last group that begins at or before the sequence
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (x.group_start[mid] <= s) lo = mid + 1; else hi = mid;
                }
                const int g = lo - 1;
                if (g >= 0 && s < clamp_to(x.group_start[g + 1], n_seq) && e.nq > 0) {
                    const Segment of = groups[g];
                    if (of.nk > 0 && e.q0 >= of.q0 && (long long)e.q0 + e.nq <= (long long)of.q0 + of.nq) {            // (bounds that do not ascend lead nowhere)
                        const int base = of.nk & ~31;
                        e.k0 = of.nk;
                        e.nk = max(e.nk - base, 0);
                        e.length -= base;
                        state = states[g];
                    }
                }
                plan.line_row[i] = s;
            }
            plan.line[i] = e;
            plan.line_state[i] = state;
            n = SharedCut::units(p, e) * p.kv_heads;
        }
        const long long run = warp_running(n);
        if (lane == 31) totals[warp] = run;
        __syncthreads();
        long long sum = before + run;
        for (int k = 0; k < PLAN_THREADS / 32; ++k) {
            if (k < warp) sum += totals[k];
            before += totals[k];
        }
        if (i < n_line) plan.unit_start[i + 1] = units[i + 1] = sum;
        __syncthreads();
    }
    if (threadIdx.x == 0) plan.unit_start[0] = units[0] = 0;
    __syncthreads();
    // where the blocks begin: each for itself would look at all of this again, one latency after the other (7 us at the start of the main kernel)
    p.line = plan.line;
    p.n_seg = n_line;
    if ((int)threadIdx.x < sms) plan.walks[threadIdx.x].begin_alone(p, units, threadIdx.x, sms);
}

// Joins the two states of every row that has two (the first blocks): a warp has one head of a row.  A state lies among the states
// where one block had its tile, else in as many parts; the parts of both are looked up at once.  Whose tile it is and which blocks had it takes
// a few dozen divisions: a block has up to SHARED_JOIN_TASKS heads of rows one behind the other, for each of whose states a thread finds out
// (when each warp did for its own, 6 groups of 8 samples of 5 tokens, 32 heads, took 20 us instead of 14).  The last blocks join the tiles of
// rows with one state that several blocks shared, as above.  (With 16 slices of each of these, which mostly have nothing to do, the kernel took
// 25 us whatever the size: eight rounds of blocks.)
constexpr int SHARED_JOIN_SLICES = 4, SHARED_JOIN_BLOCKS = 3, SHARED_JOIN_TASKS = 32;           // ... and blocks of an SM
template <typename T, int DP>
__global__ void __launch_bounds__(JOIN_WARPS * 32, SHARED_JOIN_BLOCKS) shared_join_kernel(const AttnParams p, const FwdWork w, const int sms) {
    wait_for_previous_kernel();
    const int state_blocks = (int)gridDim.x - sms * SHARED_JOIN_SLICES, behind = (int)blockIdx.x - state_blocks;
    if (behind >= 0) return join_block<T, DP>(p, w, behind / SHARED_JOIN_SLICES, behind % SHARED_JOIN_SLICES, SHARED_JOIN_SLICES);
    constexpr int E = DP / 32;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const long long units = w.unit_start[p.n_seg], blocks = Walker<SharedCut>::pieces(p, units, sms);
    struct TwoStates { int row, g, s; };                    // a row, its group (-1: it has no two states) and sequence
    struct Parts { int first, parts, r; };                  // where a state lies
    __shared__ TwoStates rows[SHARED_JOIN_TASKS];
    __shared__ Parts found[SHARED_JOIN_TASKS][2];
    const long long tasks = w.state_start[w.n_groups] * p.heads, round = (long long)SHARED_JOIN_BLOCKS * sms * JOIN_WARPS;
    const int each = JOIN_WARPS * (int)min(quotient(tasks + round - 1, round), (long long)(SHARED_JOIN_TASKS / JOIN_WARPS));        // few: a block for every eight
    for (long long base = (long long)blockIdx.x * each; base < tasks; base += (long long)state_blocks * each) {
        const int n_tasks = (int)min((long long)each, tasks - base);
        const long long at0 = quotient(base, p.heads);
        const int head0 = (int)(base - at0 * p.heads);
        __syncthreads();
        for (int k = warp; k <= (head0 + n_tasks - 1) / p.heads; k += JOIN_WARPS) {
            const int g = last_place(w.state_start, w.n_groups, at0 + k);
            const Segment shared = p.line[g];
            const long long row = at0 + k - w.line_state[g];
            TwoStates two = {0, -1, 0};
            if (shared.nq != 0 && row >= shared.q0 && row < (long long)shared.q0 + shared.nq) {
                const int a = w.first_member[g], s = a + last_place(p.q_start + a, w.n_seq - a, (int)row);
                const Segment own = p.line[w.n_groups + s];
                if (own.k0 != 0 && row >= own.q0 && row < (long long)own.q0 + own.nq) two = {(int)row, g, s};
            }
            if (lane == 0) rows[k] = two;
        }
        __syncthreads();
        if ((int)threadIdx.x < 2 * n_tasks) {
            const int k = threadIdx.x / 2, kind = threadIdx.x % 2, head = (head0 + k) % p.heads;
            const TwoStates two = rows[(head0 + k) / p.heads];
            if (two.g >= 0) {
                const int line = kind ? w.n_groups + two.s : two.g;
                const Segment seg = p.line[line];
                const int packed = (two.row - seg.q0) * p.group + head % p.group;
                const auto had = Walker<SharedCut>::blocks_of_tile(p, seg, w.unit_start[line], head / p.group, packed / FWD_ROWS, units, blocks);
                found[k][kind] = {had.first, had.parts, packed % FWD_ROWS};
            }
        }
        __syncthreads();
        for (int task = warp; task < n_tasks; task += JOIN_WARPS) {
            const int head = (head0 + task) % p.heads, ahead = (head0 + task) / p.heads, row = rows[ahead].row;
            if (rows[ahead].g < 0) continue;
            const long long at = at0 + ahead;
            const int first0 = found[task][0].first, parts0 = found[task][0].parts, r0 = found[task][0].r;
            const int first1 = found[task][1].first, parts1 = found[task][1].parts, r1 = found[task][1].r;
            // part k of both: where its maximum and mass lie, and (times DP) its accumulator
            auto place = [&](int k, const float2*& ml, const float*& o) -> long long {
                const bool kind = k >= parts0, whole = (kind ? parts1 : parts0) == 1;
                const int of = kind ? k - parts0 : k;
                ml = whole ? w.state_ml : w.part_ml;
                o = whole ? w.state_o : w.part_o;
                return whole ? ((kind ? w.state_rows : 0) + at) * p.heads + head : (2LL * ((kind ? first1 : first0) + of) + (of == 0)) * w.rows + (kind ? r1 : r0);
            };
            const int n = parts0 + parts1;
            float top = -INFINITY, mass = 0.f, o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = 0.f;
            for (int k0 = 0; k0 < n; k0 += 32) {
                const int here = min(32, n - k0);
                const float2* from_ml;
                const float* from_o;
                float2 ml = make_float2(-INFINITY, 0.f);
                if (k0 + lane < n) {
                    const long long i = place(k0 + lane, from_ml, from_o);
                    ml = from_ml[i];
                }
                float most = ml.x != ml.x ? INFINITY : ml.x;
#pragma unroll
                for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
                most = fmaxf(most, top);
                const float fade = top == -INFINITY ? 0.f : ex2(top - most), f = ml.x == -INFINITY ? 0.f : ex2(ml.x - most);
                float sum = f * ml.y;
#pragma unroll
                for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
                mass = mass * fade + sum;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] *= fade;
                top = most;
#pragma unroll 4
                for (int k = 0; k < here; ++k) {
                    const float fk = __shfl_sync(~0u, f, k);
                    const long long i = place(k0 + k, from_ml, from_o);
#pragma unroll
                    for (int e = 0; e < E; ++e) o[e] += fk * from_o[i * DP + lane + 32 * e];
                }
            }
            const long long out_row = (long long)row * p.heads + head;
            const float finish = mass > 0.f || mass != mass ? 1.f / mass : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (lane + 32 * e < p.D) ((T*)p.out)[out_row * p.D + lane + 32 * e] = Half<T>::from(finish == 0.f ? 0.f : o[e] * finish);
            if (lane == 0 && p.lse) p.lse[out_row] = mass == 0.f ? -INFINITY : (top + log2f(mass)) * LN2_F;
        }
    }
}

static size_t shared_carve(const AttnParams& p, int n_groups, void* ws, FwdWork* w, SharedPlan* plan) {
    const size_t slots = 2 * (size_t)MAX_SMS, dp = p.D > 64 ? 128 : 64, line = (size_t)n_groups + p.n_seg;
    const long long packed = (long long)p.n_q * p.group;
    w->rows = (int)(packed < FWD_ROWS ? packed : FWD_ROWS);
    w->n_groups = n_groups;
    w->n_seq = p.n_seg;
    w->state_rows = most_state_rows(p.n_seg, p.n_q, p.group);
    Carver cv(ws);
    plan->unit_start = w->unit_start = cv.take<long long>(line + 1);
    plan->line = cv.take<Segment>(line);
    plan->line_row = cv.take<int32_t>(line);
    plan->line_state = cv.take<long long>(line);
    plan->first_member = cv.take<int32_t>(n_groups);
    plan->state_start = cv.take<long long>((size_t)n_groups + 1);
    w->walks = plan->walks = cv.take<Walker<SharedCut>>(MAX_SMS);
    w->line_row = plan->line_row;
    w->line_state = plan->line_state;
    w->first_member = plan->first_member;
    w->state_start = plan->state_start;
    w->joints = cv.take<Joint>(MAX_SMS);
    w->part_ml = cv.take<float2>(slots * w->rows);
    w->part_o = cv.take<float>(slots * w->rows * dp);
    w->state_ml = cv.take<float2>(2 * (size_t)w->state_rows * p.heads);
    w->state_o = cv.take<float>(2 * (size_t)w->state_rows * p.heads * dp);
    return cv.off;
}
size_t attention_shared_bytes(const AttnParams& p, int n_groups) { FwdWork w; SharedPlan plan; return shared_carve(p, n_groups, nullptr, &w, &plan); }

template <typename T, int DP>
static tiga_status launch_shared(AttnParams p, const Prefixes& g, const FwdWork& w, const SharedPlan& plan, cudaStream_t s) {
    TileMaps maps;
    make_tile_maps(&p, operand_type<T>() == 1, &maps);
    const int sms = attention_grid();
    if (sms <= 0) return TIGA_ERR_CUDA;
    TIGA_CUDA_TRY(cudaFuncSetAttribute(attention_forward_kernel<T, DP, CUT_LINE>, cudaFuncAttributeMaxDynamicSharedMemorySize, Fwd<DP>::SMEM));
    p.item_cost = SHARED_ITEM_COST;
    p.uneven = 1;
    shared_plan_kernel<<<counted(1), PLAN_THREADS, 0, s>>>(p, g, plan, w.state_rows, sms);
    p.line = plan.line;
    p.n_seg = w.n_groups + w.n_seq;
    TIGA_CUDA_TRY(launch_after(attention_forward_kernel<T, DP, CUT_LINE>, dim3(sms), FWD_THREADS, Fwd<DP>::SMEM, s, p, w, maps));
    const long long warps = w.state_rows * p.heads, blocks = (warps + JOIN_WARPS - 1) / JOIN_WARPS, most = (long long)SHARED_JOIN_BLOCKS * sms;
    TIGA_CUDA_TRY(launch_after(shared_join_kernel<T, DP>, dim3((unsigned)(sms * SHARED_JOIN_SLICES + (blocks < most ? blocks : most))), JOIN_WARPS * 32, 0, s, p, w, sms));
    return launch_status();
}

tiga_status attention_shared(const AttnParams& p, const Prefixes& g, bool bf16, void* ws, cudaStream_t s) {
    FwdWork w;
    SharedPlan plan;
    shared_carve(p, g.n_groups, on_sectors(ws), &w, &plan);
    if (bf16) return p.D > 64 ? launch_shared<__nv_bfloat16, 128>(p, g, w, plan, s) : launch_shared<__nv_bfloat16, 64>(p, g, w, plan, s);
    return p.D > 64 ? launch_shared<__half, 128>(p, g, w, plan, s) : launch_shared<__half, 64>(p, g, w, plan, s);
}

}  // namespace tiga
