// How much attention every position of a paged cache has received: softmax weights summed over rows, on the fifth-generation tensor cores.
#include "attention_tiles.cuh"

namespace tiga {

// weight[s, h', j] = before[s, h', j] + sum over the rows i of sequence s that read position j, and the heads h of group h', of
// exp2(scale2 <q[i,h], key[j,h']> - lse2[i,h]).
// Nothing is normalised here: lse is the attention's own.  S = K Q^T lies in tensor memory with a key in every lane and a packed row of the
// group in every column; its columns are turned into weights and added up in registers, and no weight leaves them.  Sums are fp32, weights
// are never rounded to 16 bits.  A unit is 128 keys by 128 packed rows.  Of a sequence with more rows than that the keys stay (a tile, whose
// sums are put together at its end) and the rows pass by; of fewer rows the rows stay and the keys pass by, each step complete in itself, so that
// with single tokens a block reads keys without a pause.  The tile that stays and those that pass by come through a ring each.
// Four buffers of S (all of tensor memory) and four warpgroups: step n of a block belongs to buffer and warpgroup n % 4, so while one waits for
// its step or reads it, the others' exponentials run.
// What bounds it: a chunk, the exponentials (16 a cycle: 1024 cycles a unit of 1283, beside a product of 577 at a width of 128, whose operands
// come from shared memory); single tokens, the cache's keys.  2048 tokens on 16384, 32/8 heads of 128: 325 to 355 us, 282 without
// exponentials; a quarter of them by polynomials on the other pipes 360 to 423 (the warps are in order, and wait for their longer chains).
// 64 single tokens on up to 8192: 122 us, 5.7 TB/s.
constexpr int WT_WARPS = 16, WT_PRODUCER = WT_WARPS, WT_MMA = WT_PRODUCER + 4, WT_WALKER = WT_MMA + 1;
constexpr int WT_THREADS = 32 * (WT_WALKER + 1), WT_BUFFERS = 4, WT_AUX = 8;

template <int DP> struct Wt {
    static constexpr int TILE = 128 * DP * 2;
    static constexpr int STAY = 2, PASS = DP == 128 ? 4 : 8;          // tiles of the rings
    static constexpr int CONTROL = (STAY + PASS) * TILE;
    static constexpr int SMEM = CONTROL + 12 * 1024;
};
struct WtControl {
    unsigned long long x_full[2], x_empty[2], y_full[8], y_empty[8], aux_full[WT_AUX], aux_empty[WT_AUX], s_full[WT_BUFFERS], s_empty[WT_BUFFERS], drain;
    ItemRing items;
    Walker<WtCut> walk;
    uint32_t tmem, abort_word;
    alignas(16) uint32_t rows[WT_AUX][4], keys[WT_AUX][4];      // which of a step's rows and keys count
    alignas(16) float minus_lse[WT_AUX][WT_TILE];               // log2
    float share[2][4][WT_TILE];                                 // the warpgroups' sums, of alternate tiles of keys
};
static_assert(sizeof(WtControl) <= 12 * 1024, "control block");

struct WtSums {
    const float* before;            // NULL: zeros
    float* out;
    long long b_seg, b_head, o_seg, o_head, length;
};
struct WtWork {
    long long* unit_start;          // NULL: the blocks count for themselves
    Joint* joints;                  // [grid]
    float* part;                    // [2 * grid][WT_TILE]
};

__device__ __forceinline__ float weight_before(const WtSums& a, int s, int h, int j) {
    return a.before && j < a.length ? a.before[s * a.b_seg + h * a.b_head + j] : 0.f;
}
__device__ __forceinline__ void put_weight(const WtSums& a, int s, int h, int j, float v) {
    if (j < a.length) a.out[s * a.o_seg + h * a.o_head + j] = v;
}

static __global__ void __launch_bounds__(PLAN_THREADS) weights_plan_kernel(const AttnParams p, long long* unit_start) { plan_units<WtCut>(p, unit_start); }

// exp2(scale2 S - lse2) of `N` columns from column `at` on, those that `keep` has, added to sum
template <int N>
__device__ __forceinline__ f32x2 add_weights(f32x2 sum, uint32_t at, const float* minus_lse, float scale2, uint32_t keep) {
    uint32_t v[N];
    if (N == 32) tmem_ld32(at, reinterpret_cast<uint32_t(&)[32]>(v)); else tmem_ld8(at, reinterpret_cast<uint32_t(&)[8]>(v));
    if (N == 32) tmem_wait_ld(reinterpret_cast<uint32_t(&)[32]>(v)); else tmem_wait_ld(reinterpret_cast<uint32_t(&)[8]>(v));
    const float4* nl = reinterpret_cast<const float4*>(minus_lse);
    const f32x2 sc2 = dup2(scale2);
    const bool whole = __all_sync(~0u, keep == (N == 32 ? ~0u : 0xffu));
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const float4 l4 = nl[k];
        float a, b, c, d;
        unpack2(fma2(pack2(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1])), sc2, pack2(l4.x, l4.y)), a, b);
        unpack2(fma2(pack2(__uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3])), sc2, pack2(l4.z, l4.w)), c, d);
        a = ex2(a);
        b = ex2(b);
        c = ex2(c);
        d = ex2(d);
        if (!whole) {               // (a column that does not count may hold anything)
            if (!(keep >> (4 * k) & 1)) a = 0.f;
            if (!(keep >> (4 * k + 1) & 1)) b = 0.f;
            if (!(keep >> (4 * k + 2) & 1)) c = 0.f;
            if (!(keep >> (4 * k + 3) & 1)) d = 0.f;
        }
        sum = add2(sum, pack2(a, b));
        sum = add2(sum, pack2(c, d));
    }
    return sum;
}

// The same for the 128 columns of a step that count for all lanes.  A piece of 16 is on its way while one is worked on; with the last one in
// registers the buffer is free for the next product.
template <typename F>
__device__ __forceinline__ f32x2 add_step(f32x2 sum, uint32_t at, const float* minus_lse, float scale2, F free_buffer) {
    uint32_t v[2][16];
    f32x2 other = pack2(0.f, 0.f);
    const f32x2 sc2 = dup2(scale2);
    tmem_ld16(at, v[0]);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        tmem_wait_ld(v[c & 1]);
        if (c < 7) tmem_ld16(at + 16 * (c + 1), v[~c & 1]);
        else free_buffer();
        const float4* nl = reinterpret_cast<const float4*>(minus_lse + 16 * c);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 l4 = nl[k];
            float a, b, d, e;
            unpack2(fma2(pack2(__uint_as_float(v[c & 1][4 * k]), __uint_as_float(v[c & 1][4 * k + 1])), sc2, pack2(l4.x, l4.y)), a, b);
            unpack2(fma2(pack2(__uint_as_float(v[c & 1][4 * k + 2]), __uint_as_float(v[c & 1][4 * k + 3])), sc2, pack2(l4.z, l4.w)), d, e);
            sum = add2(sum, pack2(ex2(a), ex2(b)));
            other = add2(other, pack2(ex2(d), ex2(e)));
        }
    }
    return add2(sum, other);
}

template <typename T, int DP>
__global__ void __launch_bounds__(WT_THREADS, 1) attention_weights_kernel(const __grid_constant__ AttnParams p, const WtSums sums, const WtWork w, const __grid_constant__ TileMaps maps) {
    typedef Wt<DP> C;
    extern __shared__ __align__(1024) unsigned char smem[];
    WtControl& ctl = *reinterpret_cast<WtControl*>(smem + C::CONTROL);
    const uint32_t x_ring = smem_u32(smem), y_ring = x_ring + C::STAY * C::TILE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile uint32_t* abort_word = &ctl.abort_word;
    auto bar = [&](unsigned long long& b) { return smem_u32(&b); };

    wait_for_previous_kernel();
    let_next_kernel_start();
    if (threadIdx.x == 0) {
        items_init(ctl.items, WT_WALKER);
        for (int i = 0; i < C::STAY; ++i) { mbar_init(bar(ctl.x_full[i]), 32); mbar_init(bar(ctl.x_empty[i]), 1); }
        for (int i = 0; i < C::PASS; ++i) { mbar_init(bar(ctl.y_full[i]), 32); mbar_init(bar(ctl.y_empty[i]), 1); }
        for (int i = 0; i < WT_AUX; ++i) { mbar_init(bar(ctl.aux_full[i]), 1); mbar_init(bar(ctl.aux_empty[i]), 4); }
        for (int i = 0; i < WT_BUFFERS; ++i) { mbar_init(bar(ctl.s_full[i]), 1); mbar_init(bar(ctl.s_empty[i]), 128); }
        mbar_init(bar(ctl.drain), 1);
        ctl.abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == WT_WALKER) walk_begin(&ctl.walk, p, w.unit_start, blockIdx.x, gridDim.x);
    if (warp == WT_MMA) tmem_alloc(smem_u32(&ctl.tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = ctl.tmem;         // S of step n at 128 (n % WT_BUFFERS)

    if (warp == WT_WALKER) {
        if (lane == 0) {
            Walker<WtCut> walk = ctl.walk;
            w.joints[blockIdx.x] = joint_of(p, walk, walk.here && !WtCut::narrow(p, walk.g), blockIdx.x);
            items_hand_out(ctl.items, p, walk, walk.here);
        }
        __syncwarp();
    } else if (warp >= WT_PRODUCER && warp < WT_MMA) {
        // ---------------------------------------------------------------- producers: step n is that of warp n % 4, tiles that stay are the first's
        // Whatever lies in a key's or a row's place reaches that key's lane, or that row's column, alone, and those that do not count are left
        // out of the sums.  So boxes bring whole groups of rows, with what lies behind the last one; only pages that are missing are not asked for.
        const int pw = warp - WT_PRODUCER;
        uint32_t items = 0, steps = 0, last = 0;        // tiles that stay; steps of the items before; one behind this warp's last step
        bool ok = true;
        auto wait = [&](unsigned long long& b, uint32_t parity) { return ok = __all_sync(~0u, mbar_wait(bar(b), parity & 1, abort_word)); };
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const Segment g = e.segment();
            const bool narrow = WtCut::narrow(p, g);
            const int skip = WtCut::skipped(p, g, e.t), i0 = e.i0 + skip, n = e.i1 - e.i0, h = e.h, packed = g.nq * p.group;
            // key tile or row tile number i: where the lane's four keys lie, and which of all there are; its rows' lse (-inf: there is none, or it
            // reads nothing)
            Place at[4];
            uint32_t there[4];
            float lse[4];
            auto look_keys = [&](int i) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int j = i * WT_TILE + 32 * c + lane;
                    at[c] = j < g.nk && g.nq ? key_place(p, g, e.s, j) : Place{-1, 0};
                }
            };
            auto look_rows = [&](int i) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int r = i * WT_TILE + 32 * c + lane;
                    lse[c] = -INFINITY;
                    if (r < packed) {
                        const PackedRow pr = packed_row(p, g, h, r);
                        lse[c] = p.lse_in[(long long)pr.row * p.heads + pr.head];
                    }
                }
            };
            auto vote_keys = [&]() {
#pragma unroll
                for (int c = 0; c < 4; ++c) there[c] = __ballot_sync(~0u, at[c].at >= 0);
            };
            auto fetch_key_tile = [&](uint32_t tile, uint32_t full) {
                if (p.kv_box) {
                    const uint32_t first = p.kv_box == 32 ? 1u : p.kv_box == 16 ? 0x10001u : 0x1010101u;            // lanes at which a box begins
                    int boxes = 0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) boxes += __popc(there[c] & first);
                    if (lane == 0) { mbar_arrive(full, 31); mbar_arrive_expect(full, boxes * p.kv_box * DP * 2); }
                    __syncwarp();
                    if (first >> lane & 1)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (at[c].at >= 0)
#pragma unroll
                                for (int f = 0; f < DP / 64; ++f) box_copy(tile + f * (128 * 128) + (32 * c + lane) * 128, &maps.k, full, 64 * f, at[c].slot, h, at[c].at);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) copy_rows<DP, 128, 32>(tile, 32 * c, p.k, key_offset(p, at[c], h), p.D, w.part);
                    cp_async_arrive(full);
                }
            };
            auto fetch_row_tile = [&](int i, uint32_t tile, uint32_t full) {
                if (p.q_box) {
                    if (lane == 0) { mbar_arrive(full, 31); mbar_arrive_expect(full, 128 * DP * 2); }
                    __syncwarp();
                    if (lane < DP / 64) box_copy(tile + lane * (128 * 128), &maps.q, full, 64 * lane, h * p.group, g.q0 + i * (WT_TILE / p.group), 0);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int r = i * WT_TILE + 32 * c + lane;
                        const PackedRow pr = packed_row(p, g, h, r < packed ? r : 0);
                        if (i * WT_TILE + 32 * c < packed) copy_rows<DP, 128, 32>(tile, 32 * c, p.q, r < packed ? pr.row * p.q_row + pr.head * p.q_head : -1, p.D, w.part);
                    }
                    cp_async_arrive(full);
                }
            };
            if (narrow) look_rows(0);
            else { look_keys(e.t); vote_keys(); }
            if (pw == 0 && ok) {
                const uint32_t stay = item % C::STAY, tile = x_ring + stay * C::TILE, full = bar(ctl.x_full[stay]);
                if (item < (uint32_t)C::STAY || wait(ctl.x_empty[stay], item / C::STAY + 1)) {
                    if (narrow) fetch_row_tile(0, tile, full); else fetch_key_tile(tile, full);
                    ++items;
                }
            }
            for (int i = (int)((pw - steps) % 4); i < n && ok; i += 4) {
                const uint32_t step = steps + i, slot = step % C::PASS, aux = step % WT_AUX;
                if (narrow) look_keys(i0 + i); else look_rows(i0 + i);
                if (step >= (uint32_t)C::PASS && !wait(ctl.y_empty[slot], step / C::PASS + 1)) break;
                const uint32_t tile = y_ring + slot * C::TILE, full = bar(ctl.y_full[slot]);
                if (narrow) { vote_keys(); fetch_key_tile(tile, full); }
                else fetch_row_tile(i0 + i, tile, full);
                last = step + 1;
                if (step >= (uint32_t)WT_AUX && !wait(ctl.aux_empty[aux], step / WT_AUX + 1)) break;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t valid = __ballot_sync(~0u, lse[c] != -INFINITY);
                    ctl.minus_lse[aux][32 * c + lane] = lse[c] == -INFINITY ? 0.f : -lse[c] * LOG2E_F;
                    if (lane == 0) { ctl.rows[aux][c] = valid; ctl.keys[aux][c] = there[c]; }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.aux_full[aux]));
            }
            steps += n;
            item_return(ctl.items, item);
        }
        cp_async_wait_all();
        if (*abort_word) {          // boxes may still be on their way: the tiles that this warp asked for
            for (uint32_t k = items < (uint32_t)C::STAY ? 0 : items - C::STAY; k < items; ++k) mbar_wait_for(bar(ctl.x_full[k % C::STAY]), (k / C::STAY) & 1, HALF_A_SECOND);
            for (uint32_t k = last; k > 0 && last - k < (uint32_t)C::PASS; k -= min(k, 4u)) mbar_wait_for(bar(ctl.y_full[(k - 1) % C::PASS]), ((k - 1) / C::PASS) & 1, HALF_A_SECOND);
        }
    } else if (warp == WT_MMA) {
        // ---------------------------------------------------------------- matrix instructions
        const uint32_t sign = p.scale < 0.f ? MMA_NEGATE_A : 0, x_desc = smem_desc(x_ring, 16), y_desc = smem_desc(y_ring, 16);
        uint32_t steps = 0;
        bool ok = true;
        auto wait = [&](unsigned long long& b, uint32_t parity) { ok = __all_sync(~0u, ok && mbar_wait(bar(b), parity & 1, abort_word)); };
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const bool narrow = WtCut::narrow(p, e.segment());
            const int skip = WtCut::skipped(p, e.segment(), e.t), i0 = e.i0 + skip, i1 = e.i1 + skip, packed = e.nq * p.group;
            item_return(ctl.items, item);
            if (!ok) continue;
            const uint32_t stay = item % C::STAY;
            wait(ctl.x_full[stay], item / C::STAY);
            for (int i = i0; i < i1 && ok; ++i, ++steps) {
                const uint32_t buffer = steps % WT_BUFFERS, slot = steps % C::PASS;
                const int columns = narrow ? packed : min(packed - i * WT_TILE, WT_TILE);
                const uint32_t shape = mma_shape<T>(max((columns + 15) & ~15, 16), false) | sign;
                wait(ctl.y_full[slot], steps / C::PASS);
                if (steps >= (uint32_t)WT_BUFFERS) { wait(ctl.s_empty[buffer], steps / WT_BUFFERS + 1); tmem_fence_after(); }
                if (!ok) break;
                fence_async_proxy();
                const uint32_t x = x_desc + stay * (C::TILE / 16), y = y_desc + slot * (C::TILE / 16), k = narrow ? y : x, q = narrow ? x : y;
                if (elected()) {
#pragma unroll
                    for (int c = 0; c < DP / 16; ++c)
                        if (c * 16 < p.D) mma_ss(tmem + 128 * buffer, k + piece(c), q + piece(c), shape, c > 0);
                    mma_commit(bar(ctl.s_full[buffer]));
                    mma_commit(bar(ctl.y_empty[slot]));
                    if (i + 1 == i1) mma_commit(bar(ctl.x_empty[stay]));
                }
                __syncwarp();
            }
        }
        if (elected()) mma_commit(bar(ctl.drain));
        mbar_wait_for(bar(ctl.drain), 0, HALF_A_SECOND);
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- weights: a key a thread
        const int x = warp / 4, row = threadIdx.x & 127;
        const uint32_t S = tmem + ((uint32_t)(warp % 4 * 32) << 16) + 128 * x;
        const float scale2 = fmaxf(fabsf(p.scale) * LOG2E_F, 1e-30f);
        uint32_t steps = 0, wide = 0;               // steps of the items before; tiles of keys so far
        bool ok = true;
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const Segment g = e.segment();
            const bool narrow = WtCut::narrow(p, g);
            const int skip = WtCut::skipped(p, g, e.t), n = e.i1 - e.i0, packed = g.nq * p.group, before = g.length - g.nq;
            const bool whole_tile = n == e.steps;
            const int key = e.t * WT_TILE + row;            // wide: this thread's key
            const float base = !narrow && whole_tile && x == 0 && key < g.nk ? weight_before(sums, e.s, e.h, key) : 0.f;
            f32x2 sum = pack2(0.f, 0.f);
            uint32_t there = 0;             // the keys of this warp that there are (wide: as the last step says; all say the same)
            for (int i = (int)((x - steps) % WT_BUFFERS); i < n; i += WT_BUFFERS) {
                const uint32_t step = steps + i, aux = step % WT_AUX;
                const int tile = e.i0 + skip + i, j = narrow ? tile * WT_TILE + row : key;
                const float old = narrow && j < g.nk ? weight_before(sums, e.s, e.h, j) : 0.f;
                // under the triangle: columns in front of the first row that reads this key
                const int edge = p.causal ? min(max(j - before, 0), g.nq) * p.group - (narrow ? 0 : tile * WT_TILE) : 0;
                const int columns = narrow ? packed : min(packed - tile * WT_TILE, WT_TILE);
                ok = ok && mbar_wait(bar(ctl.aux_full[aux]), (step / WT_AUX) & 1, abort_word) && mbar_wait(bar(ctl.s_full[x]), (step / WT_BUFFERS) & 1, abort_word);
                ok = __all_sync(~0u, ok);
                tmem_fence_after();
                const uint4 rows = *reinterpret_cast<const uint4*>(ctl.rows[aux]);
                const bool all = __all_sync(~0u, edge <= 0) && columns == WT_TILE && (rows.x & rows.y & rows.z & rows.w) == ~0u;
                auto free_buffer = [&]() {
                    tmem_fence_before();
                    mbar_arrive(bar(ctl.s_empty[x]));
                };
                if (ok) there = ctl.keys[aux][warp % 4];
                if (ok && all) sum = add_step(sum, S, ctl.minus_lse[aux], scale2, free_buffer);
                else {
                    if (ok)
#pragma unroll 1
                        for (int c = 0; 32 * c < columns; ++c) {
                            const int cut = edge - 32 * c;
                            const uint32_t keep = ctl.rows[aux][c] & (cut <= 0 ? ~0u : cut >= 32 ? 0u : ~0u << cut);
                            if (columns - 32 * c > 8) sum = add_weights<32>(sum, S + 32 * c, ctl.minus_lse[aux] + 32 * c, scale2, keep);
                            else sum = add_weights<8>(sum, S + 32 * c, ctl.minus_lse[aux] + 32 * c, scale2, keep & 0xff);
                        }
                    free_buffer();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.aux_empty[aux]));
                if (narrow) {               // complete
                    float a, b;
                    unpack2(sum, a, b);
                    a = there >> lane & 1 ? a + b : 0.f;
                    if (j < g.nk) put_weight(sums, e.s, e.h, j, ok ? old + a : __int_as_float(0x7fffffff));
                    sum = pack2(0.f, 0.f);
                }
            }
            if (!narrow) {
                float a, b;
                unpack2(sum, a, b);
                a = there >> lane & 1 ? a + b : 0.f;
                // (a buffer is written again two tiles of keys later, behind the meeting of the one in between)
                ctl.share[wide & 1][x][row] = ok ? a : __int_as_float(0x7fffffff);
                asm volatile("bar.sync 1, 512;" ::: "memory");
                if (x == 0 && key < g.nk) {
                    float total = 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) total += ctl.share[wide & 1][k][row];
                    if (whole_tile) put_weight(sums, e.s, e.h, key, base + total);
                    else w.part[(2LL * blockIdx.x + (e.i0 == 0)) * WT_TILE + row] = total;
                }
                ++wide;
            }
            steps += n;
            item_return(ctl.items, item);
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == WT_MMA) { tmem_fence_after(); tmem_free(tmem, 512); }
}

// Adds up the partial sums of a tile that several blocks shared, in the order of its steps.
static __global__ void __launch_bounds__(WT_TILE) weights_sum_kernel(const AttnParams p, const WtSums sums, const WtWork w) {
    wait_for_previous_kernel();
    const Joint& j = w.joints[blockIdx.x];
    if (j.parts == 0) return;
    const int row = threadIdx.x, key = j.item.t * WT_TILE + row;
    if (key >= j.item.nk) return;
    float sum = 0.f;
#pragma unroll 8
    for (int k = 0; k < j.parts; ++k) sum += w.part[(2LL * (j.first + k) + (k == 0)) * WT_TILE + row];
    put_weight(sums, j.item.s, j.item.h, key, weight_before(sums, j.item.s, j.item.h, key) + sum);
}

// A sequence may be longer than its row of the table: entries of the positions from `room` on, which receive nothing, are what was before.  By
// pieces of a list.
constexpr int REST_THREADS = 256, REST_PIECE = 16 * REST_THREADS;
static __global__ void __launch_bounds__(REST_THREADS) weights_rest_kernel(const AttnParams p, const WtSums sums, const long long room, const long long pieces) {
    const long long tasks = (long long)p.n_seg * p.kv_heads * pieces;
    for (long long task = blockIdx.x; task < tasks; task += gridDim.x) {
        const long long list = quotient(task, pieces), first = room + (task - list * pieces) * REST_PIECE;
        const int s = (int)quotient(list, p.kv_heads), h = (int)(list - (long long)s * p.kv_heads);
        const long long end = min(min((long long)p.kv_len[s], sums.length), first + REST_PIECE);
        for (long long j = first + threadIdx.x; j < end; j += REST_THREADS) put_weight(sums, s, h, (int)j, weight_before(sums, s, h, (int)j));
    }
}

static size_t weights_carve(const AttnParams& p, void* ws, WtWork* w) {
    Carver cv(ws);
    w->unit_start = cv.take<long long>((size_t)p.n_seg + 1);
    if (counts_itself(p, WT_TILE, true)) w->unit_start = nullptr;
    w->joints = cv.take<Joint>(MAX_SMS);
    w->part = cv.take<float>(2 * (size_t)MAX_SMS * WT_TILE);
    return cv.off;
}

template <typename T, int DP>
static tiga_status launch_weights(AttnParams p, const WtSums& sums, const WtWork& w, cudaStream_t s) {
    TileMaps maps;
    make_tile_maps(&p, operand_type<T>() == 1, &maps);
    p.q_box = make_row_map(p, operand_type<T>() == 1, WT_TILE, &maps.q) ? WT_TILE : 0;
    const int sms = attention_grid();
    if (sms <= 0) return TIGA_ERR_CUDA;
    TIGA_CUDA_TRY(cudaFuncSetAttribute(attention_weights_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Wt<DP>::SMEM));
    if (w.unit_start) {
        weights_plan_kernel<<<counted(1), PLAN_THREADS, 0, s>>>(p, w.unit_start);
        TIGA_CUDA_TRY(launch_after(attention_weights_kernel<T, DP>, dim3(sms), WT_THREADS, Wt<DP>::SMEM, s, p, sums, w, maps));
    } else attention_weights_kernel<T, DP><<<counted((unsigned)sms), WT_THREADS, Wt<DP>::SMEM, s>>>(p, sums, w, maps);
    // no sequence has more than n_q rows: if those are few, no sum is in parts
    if ((long long)p.n_q * p.group > WT_TILE) TIGA_CUDA_TRY(launch_after(weights_sum_kernel, dim3(sms), WT_TILE, 0, s, p, sums, w));
    return launch_status();
}

}  // namespace tiga

using namespace tiga;

extern "C" size_t tiga_paged_weights_workspace_bytes(const tiga_pages* c, const tiga_heads* h, int64_t n_q) {
    AttnParams p;
    if (attention_paged_check(c, h, n_q, &p) != TIGA_OK) return 0;
    WtWork w;
    return weights_carve(p, nullptr, &w) + 256;
}

extern "C" tiga_status tiga_paged_attention_weights(const tiga_pages* c, const tiga_heads* h, const void* q, const int32_t* q_start, int64_t n_q,
                                                    const float* lse, int causal, const tiga_weights* before, const tiga_weights* weights,
                                                    void* ws, size_t ws_bytes, void* stream) {
    AttnParams p;
    tiga_status st = attention_paged_check(c, h, n_q, &p);
    if (st != TIGA_OK) return st;
    if (attention_bad_stride(h->q) || attention_bad_weights(weights) || (before && (attention_bad_weights(before) || before->length < weights->length))) return TIGA_ERR_INVALID_ARG;
    if (c->n_seg == 0 || weights->length == 0) return TIGA_OK;
    if (attention_bad_ints(q_start) || attention_bad_ints(c->kv_len) || !aligned16(weights->data) || !weights->data) return TIGA_ERR_INVALID_ARG;
    if (attention_weights_overlap(weights, c->n_seg, h->kv_heads)) return TIGA_ERR_INVALID_ARG;
    if (before && (!before->data || !aligned16(before->data))) return TIGA_ERR_INVALID_ARG;
    if (before && before->data == weights->data && ((c->n_seg > 1 && before->seg != weights->seg) || (h->kv_heads > 1 && before->head != weights->head))) return TIGA_ERR_INVALID_ARG;
    if (n_q > 0 && (!q || !aligned16(q) || !lse || !aligned16(lse))) return TIGA_ERR_INVALID_ARG;
    if ((c->max_pages > 0 && attention_bad_ints(c->table)) || (c->n_pages > 0 && (!c->key || !aligned16(c->key)))) return TIGA_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < tiga_paged_weights_workspace_bytes(c, h, n_q)) return TIGA_ERR_WORKSPACE;
    if (c->max_pages == 0 && !before) return TIGA_OK;           // neither positions nor what they had before
    const WtSums sums = {before ? before->data : nullptr, weights->data, before ? before->seg : 0, before ? before->head : 0, weights->seg, weights->head, weights->length};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long room = c->max_pages * c->page_size;
    if (room < sums.length && sums.before != sums.out) {
        const long long pieces = (sums.length - room + REST_PIECE - 1) / REST_PIECE, tasks = c->n_seg * h->kv_heads * pieces;
        weights_rest_kernel<<<counted((unsigned)(tasks < 4096 ? tasks : 4096)), REST_THREADS, 0, s>>>(p, sums, room, pieces);
    }
    if (c->max_pages == 0) return launch_status();
    WtWork w;
    weights_carve(p, ws, &w);
    p.q = q; p.v = p.k; p.q_start = q_start; p.causal = causal != 0; p.lse_in = lse;
    if (h->dtype == TIGA_BF16) return p.D > 64 ? launch_weights<__nv_bfloat16, 128>(p, sums, w, s) : launch_weights<__nv_bfloat16, 64>(p, sums, w, s);
    return p.D > 64 ? launch_weights<__half, 128>(p, sums, w, s) : launch_weights<__half, 64>(p, sums, w, s);
}
