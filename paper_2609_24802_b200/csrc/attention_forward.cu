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
// What bounds it: the chain S -> maximum -> P -> O of a half, 4050 cycles a step of 128 keys at a width of 128 where its products take
// 1024 and its 16384 exponentials another 1024.  Two threads a row halve what one would take (a warp alone on its scheduler needs
// about 13 cycles a column); the exchange of their maxima costs 100.  4 segments of 4096 rows and keys, 16/4 heads of 128, bf16: 543 us
// alone, 1.0 PFLOP/s; single tokens read their cache at 6.3 TB/s between the ends of items.
constexpr int FWD_SOFTMAX_WARPS = 16, FWD_PRODUCER = FWD_SOFTMAX_WARPS, FWD_MMA = FWD_PRODUCER + 4, FWD_WALKER = FWD_MMA + 1;
constexpr int FWD_THREADS = 32 * (FWD_WALKER + 1), FWD_ROWS = 256, FWD_STEP = 128;
typedef Cut<FWD_ROWS, FWD_STEP, false> FwdCut;
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
};

static __global__ void __launch_bounds__(PLAN_THREADS) forward_plan_kernel(const AttnParams p, long long* unit_start) { plan_units<FwdCut>(p, unit_start); }

template <typename T, int DP>
__global__ void __launch_bounds__(FWD_THREADS, 1) attention_forward_kernel(const AttnParams p, const FwdWork w, const __grid_constant__ TileMaps maps) {
    typedef Fwd<DP> C;
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
    Walker<FwdCut> walk;
    bool work_here = false;
    if (warp == FWD_WALKER) work_here = walk.begin(p, w.unit_start, blockIdx.x, gridDim.x);
    if (warp == FWD_MMA) tmem_alloc(smem_u32(&ctl.tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = ctl.tmem;
    // tensor memory: S of half x at 128 x, O at 256 + DP x

    if (warp == FWD_WALKER) {
        if (lane == 0) {
            w.joints[blockIdx.x] = joint_of(walk, work_here, blockIdx.x);
            items_hand_out(ctl.items, p, walk, work_here);
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
            const int i0 = e.i0, i1 = e.i1, h = e.h;
            auto place = [&](int i) {
                const int j = i * FWD_STEP + 32 * pw + lane;
                return j < g.nk ? key_place(p, g, e.s, j) : Place{-1, 0};
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
            const bool whole_tile = n == e.steps;
            const long long part = (2LL * blockIdx.x + (e.i0 == 0)) * w.rows + tile_row;
            const PackedRow pr = packed_row(p, e.segment(), e.h, e.t * FWD_ROWS + tile_row);
            const long long out_row = (long long)pr.row * p.heads + pr.head;
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
                        store_rows<2>(o, (T*)p.out + out_row * p.D + f, valid, (p.D - f) / 8);
                    } else if (valid) {
                        uint4* out = reinterpret_cast<uint4*>(w.part_o + part * DP + f);
#pragma unroll
                        for (int k = 0; k < 4; ++k) out[k] = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                    }
                }
            if (valid && y == 0 && (two || x == 0)) {
                if (!whole_tile) w.part_ml[part] = make_float2(m - BIAS, l);
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

template <typename T, int DP>
__global__ void __launch_bounds__(JOIN_WARPS * 32) attention_join_kernel(const AttnParams p, const FwdWork w) {
    wait_for_previous_kernel();
    const Joint& j = w.joints[blockIdx.x];
    const int parts = j.parts;
    if (parts == 0) return;
    const Item it = j.item;
    const int first = j.first, rows = min(it.nq * p.group - it.t * FWD_ROWS, FWD_ROWS);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    constexpr int E = DP / 32;
    __shared__ float sh_m[JOIN_WARPS], sh_l[JOIN_WARPS], sh_o[JOIN_WARPS][DP];
    const bool few = parts <= JOIN_FEW;
    for (int r = few ? blockIdx.y * JOIN_WARPS + warp : blockIdx.y; r < rows; r += few ? JOIN_Y * JOIN_WARPS : JOIN_Y) {
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

size_t attention_forward_carve(const AttnParams& p, void* ws, FwdWork* w) {
    const size_t slots = 2 * (size_t)MAX_SMS;
    const long long packed = (long long)p.n_q * p.group;
    w->rows = (int)(packed < FWD_ROWS ? packed : FWD_ROWS);
    Carver cv(ws);
    w->unit_start = cv.take<long long>((size_t)p.n_seg + 1);       // (room for it whether or not this call needs it: its size is asked for without `causal`)
    if (counts_itself(p, FWD_ROWS)) w->unit_start = nullptr;
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
    TIGA_CUDA_TRY(cudaFuncSetAttribute(attention_forward_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Fwd<DP>::SMEM));
    if (w.unit_start) forward_plan_kernel<<<counted(1), PLAN_THREADS, 0, s>>>(p, w.unit_start);
    if (w.unit_start) TIGA_CUDA_TRY(launch_after(attention_forward_kernel<T, DP>, dim3(sms), FWD_THREADS, Fwd<DP>::SMEM, s, p, w, maps));
    else attention_forward_kernel<T, DP><<<counted((unsigned)sms), FWD_THREADS, Fwd<DP>::SMEM, s>>>(p, w, maps);
    TIGA_CUDA_TRY(launch_after(attention_join_kernel<T, DP>, dim3(sms, JOIN_Y), JOIN_WARPS * 32, 0, s, p, w));
    return launch_status();
}

tiga_status attention_forward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s) {
    FwdWork w;
    attention_forward_carve(p, ws, &w);
    if (bf16) return p.D > 64 ? launch_forward<__nv_bfloat16, 128>(p, w, s) : launch_forward<__nv_bfloat16, 64>(p, w, s);
    return p.D > 64 ? launch_forward<__half, 128>(p, w, s) : launch_forward<__half, 64>(p, w, s);
}

}  // namespace tiga
