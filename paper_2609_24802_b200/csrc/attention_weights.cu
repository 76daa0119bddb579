// How much attention every position of a paged cache has received: softmax weights summed over rows, on the fifth-generation tensor cores.
#include "attention_tiles.cuh"

namespace tiga {

// weight[s, h', j] = before[s, h', j] + sum over the rows i of sequence s that read position j, and the heads h of group h', of
// exp2(scale2 <q[i,h], key[j,h']> - lse2[i,h]).
// Nothing is normalised here: lse is the attention's own.  So keys are stationary (a tile of 128) and the packed rows of a group pass by in
// steps of 128: S = K Q^T lies in tensor memory with a key in every lane, its columns are turned into weights and added up in registers,
// and no weight leaves them.  Four S buffers (all of tensor memory) let the products run ahead.  The keys' tiles come through a ring of
// their own, so that those of the next items are on their way while one is worked on; so do the rows'.
// A step with few rows is as narrow as they are (16 columns at least).  Sums are fp32, weights are never rounded to 16 bits.
// What bounds it: a chunk, the exponentials (16 a cycle: 1024 cycles a step of 128 x 128, whose product takes 256 at a width of 128);
// single tokens, the cache's keys.
constexpr int WT_WARPS = 16, WT_PRODUCER = WT_WARPS, WT_MMA = WT_PRODUCER + 4, WT_WALKER = WT_MMA + 1;
constexpr int WT_THREADS = 32 * (WT_WALKER + 1), WT_TILE = 128, WT_STEP = 128, WT_BUFFERS = 4;
typedef Cut<WT_TILE, WT_STEP, true> WtCut;

template <int DP> struct Wt {
    static constexpr int TILE = 128 * DP * 2;
    static constexpr int KEYS = DP == 128 ? 3 : 6, ROWS = DP == 128 ? 3 : 6;       // tiles of the rings
    static constexpr int CONTROL = (KEYS + ROWS) * TILE;
    static constexpr int SMEM = CONTROL + 7 * 1024;
};
struct WtControl {
    unsigned long long k_full[6], k_empty[6], q_full[6], q_empty[6], aux_full[WT_BUFFERS], s_full[WT_BUFFERS], s_empty[WT_BUFFERS], drain;
    ItemRing items;
    Walker<WtCut> walk;
    uint32_t tmem, abort_word, mask[WT_BUFFERS][4];             // which of a step's rows count
    uint32_t keys[ITEMS][4];                                    // which of an item's keys there are (an item's place is free once all warps returned it)
    alignas(16) float minus_lse[WT_BUFFERS][WT_STEP];           // log2
    float share[2][3][WT_TILE];                                 // sums of the second to fourth warpgroup, of alternate wide items
};
static_assert(sizeof(WtControl) <= 7 * 1024, "control block");

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

template <typename T, int DP>
__global__ void __launch_bounds__(WT_THREADS, 1) attention_weights_kernel(const __grid_constant__ AttnParams p, const WtSums sums, const WtWork w, const __grid_constant__ TileMaps maps) {
    typedef Wt<DP> C;
    extern __shared__ __align__(1024) unsigned char smem[];
    WtControl& ctl = *reinterpret_cast<WtControl*>(smem + C::CONTROL);
    const uint32_t keys = smem_u32(smem), rows = keys + C::KEYS * C::TILE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile uint32_t* abort_word = &ctl.abort_word;
    auto bar = [&](unsigned long long& b) { return smem_u32(&b); };

    wait_for_previous_kernel();
    let_next_kernel_start();
    if (threadIdx.x == 0) {
        items_init(ctl.items, WT_WALKER);
        for (int i = 0; i < C::KEYS; ++i) { mbar_init(bar(ctl.k_full[i]), 128); mbar_init(bar(ctl.k_empty[i]), 1); }
        for (int i = 0; i < C::ROWS; ++i) { mbar_init(bar(ctl.q_full[i]), 128); mbar_init(bar(ctl.q_empty[i]), 1); }
        for (int i = 0; i < WT_BUFFERS; ++i) {
            mbar_init(bar(ctl.aux_full[i]), 4);
            mbar_init(bar(ctl.s_full[i]), 1);
            mbar_init(bar(ctl.s_empty[i]), 32 * WT_WARPS);
        }
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
    // rows of step i (of all steps of the segment) that exist
    auto rows_of = [&](const Item& e, int i) { return min(max(e.nq * p.group - i * WT_STEP, 0), WT_STEP); };

    if (warp == WT_WALKER) {
        if (lane == 0) {
            Walker<WtCut> walk = ctl.walk;
            w.joints[blockIdx.x] = joint_of(walk, walk.here, blockIdx.x);
            items_hand_out(ctl.items, p, walk, walk.here);
        }
        __syncwarp();
    } else if (warp >= WT_PRODUCER && warp < WT_MMA) {
        // ---------------------------------------------------------------- producers
        const int pw = warp - WT_PRODUCER;
        uint32_t items = 0, steps = 0;          // tiles of keys, and of rows, that were asked for
        bool ok = true;
        auto wait = [&](unsigned long long& b, uint32_t parity) { return ok = __all_sync(~0u, mbar_wait(bar(b), parity & 1, abort_word)); };
        // Where the keys of an item and the rows of a step lie comes from global memory: looked up one item and one step ahead.
        auto place = [&](const Item& e) {
            const int j = e.t * WT_TILE + 32 * pw + lane;
            return j < e.nk && e.nq ? key_place(p, e.segment(), e.s, j) : Place{-1, 0};
        };
        auto look = [&](const Item& e, int i) {
            const int r = i * WT_STEP + 32 * pw + lane;
            if (r >= e.nq * p.group) return -INFINITY;
            const PackedRow pr = packed_row(p, e.segment(), e.h, r);
            return p.lse_in[(long long)pr.row * p.heads + pr.head];
        };
        const Item* e = &item_take(ctl.items, 0);
        Place at{-1, 0};
        float lse = -INFINITY;
        if (e->steps) { at = place(*e); lse = look(*e, e->i0 + WtCut::skipped(p, e->segment(), e->t)); }
        for (uint32_t item = 0; e->steps; ++item) {
            const Segment g = e->segment();
            const int skip = WtCut::skipped(p, g, e->t), i0 = e->i0 + skip, i1 = ok ? e->i1 + skip : i0, h = e->h;
            const Item* next = &item_take(ctl.items, item + 1);
            const Place here = at;
            if (next->steps) at = place(*next);
            const uint32_t there = __ballot_sync(~0u, here.at >= 0);
            if (lane == 0) ctl.keys[item % ITEMS][pw] = there;              // (seen behind aux_full of the item's first step)
            if (ok && (item < (uint32_t)C::KEYS || wait(ctl.k_empty[item % C::KEYS], item / C::KEYS + 1))) {
                fetch_keys<DP>(keys + (item % C::KEYS) * C::TILE, 32 * pw, bar(ctl.k_full[item % C::KEYS]), p, maps, false, here, h, w.part);
                ++items;
            }
            for (int i = i0; i < i1 && ok; ++i) {
                const int r = i * WT_STEP + 32 * pw + lane, buffer = steps % WT_BUFFERS;
                const float mine = lse;
                if (i + 1 < i1) lse = look(*e, i + 1);
                else if (next->steps) lse = look(*next, next->i0 + WtCut::skipped(p, next->segment(), next->t));
                const uint32_t slot = steps % C::ROWS, tile = rows + slot * C::TILE, full = bar(ctl.q_full[slot]);
                if (steps >= (uint32_t)C::ROWS && !wait(ctl.q_empty[slot], steps / C::ROWS + 1)) break;
                if (32 * pw < rows_of(*e, i)) fetch_packed<DP>(tile, 32 * pw, full, p, g, maps, false, h, r, mine != -INFINITY, w.part);
                else if (lane == 0) mbar_arrive(full, 32);
                const uint32_t step = steps++;
                if (step >= (uint32_t)WT_BUFFERS && !wait(ctl.s_empty[buffer], step / WT_BUFFERS + 1)) break;
                const uint32_t valid = __ballot_sync(~0u, mine != -INFINITY);       // (a row that reads nothing counts nowhere, whatever its query holds)
                ctl.minus_lse[buffer][32 * pw + lane] = mine == -INFINITY ? 0.f : -mine * LOG2E_F;
                if (lane == 0) ctl.mask[buffer][pw] = valid;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.aux_full[buffer]));
            }
            item_return(ctl.items, item);
            e = next;
        }
        cp_async_wait_all();
        if (*abort_word) {          // boxes may still be on their way: their tiles, as far as they were asked for
            for (uint32_t k = items < (uint32_t)C::KEYS ? 0 : items - C::KEYS; k < items; ++k) mbar_wait_for(bar(ctl.k_full[k % C::KEYS]), (k / C::KEYS) & 1, HALF_A_SECOND);
            for (uint32_t k = steps < (uint32_t)C::ROWS ? 0 : steps - C::ROWS; k < steps; ++k) mbar_wait_for(bar(ctl.q_full[k % C::ROWS]), (k / C::ROWS) & 1, HALF_A_SECOND);
        }
    } else if (warp == WT_MMA) {
        // ---------------------------------------------------------------- matrix instructions
        const uint32_t sign = p.scale < 0.f ? MMA_NEGATE_A : 0, k_desc = smem_desc(keys, 16), q_desc = smem_desc(rows, 16);
        uint32_t steps = 0;
        bool ok = true;
        auto wait = [&](unsigned long long& b, uint32_t parity) { ok = __all_sync(~0u, ok && mbar_wait(bar(b), parity & 1, abort_word)); };
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const int skip = WtCut::skipped(p, e.segment(), e.t), i0 = e.i0 + skip, i1 = e.i1 + skip, packed = e.nq * p.group;
            item_return(ctl.items, item);
            if (!ok) continue;
            const uint32_t k_slot = item % C::KEYS;
            wait(ctl.k_full[k_slot], item / C::KEYS);
            for (int i = i0; i < i1 && ok; ++i, ++steps) {
                const uint32_t buffer = steps % WT_BUFFERS, q_slot = steps % C::ROWS, columns = min(max(packed - i * WT_STEP, 0), WT_STEP);
                const uint32_t shape = mma_shape<T>(max((columns + 15) & ~15, 16), false) | sign;
                wait(ctl.q_full[q_slot], steps / C::ROWS);
                if (steps >= (uint32_t)WT_BUFFERS) { wait(ctl.s_empty[buffer], steps / WT_BUFFERS + 1); tmem_fence_after(); }
                if (!ok) break;
                fence_async_proxy();
                const uint32_t k = k_desc + k_slot * (C::TILE / 16), q = q_desc + q_slot * (C::TILE / 16);
                if (elected()) {
#pragma unroll
                    for (int c = 0; c < DP / 16; ++c)
                        if (c * 16 < p.D) mma_ss(tmem + 128 * buffer, k + piece(c), q + piece(c), shape, c > 0);
                    mma_commit(bar(ctl.s_full[buffer]));
                    mma_commit(bar(ctl.q_empty[q_slot]));
                    if (i + 1 == i1) mma_commit(bar(ctl.k_empty[k_slot]));
                }
                __syncwarp();
            }
        }
        if (elected()) mma_commit(bar(ctl.drain));
        mbar_wait_for(bar(ctl.drain), 0, HALF_A_SECOND);
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- weights: a key a thread, warpgroup x has 32 of a step's 128 columns
        const int x = warp / 4, row = threadIdx.x & 127;
        const uint32_t S = tmem + ((uint32_t)(warp % 4 * 32) << 16) + 32 * x;
        const float scale2 = fmaxf(fabsf(p.scale) * LOG2E_F, 1e-30f);
        const f32x2 sc2 = dup2(scale2);
        uint32_t steps = 0, wide = 0;
        bool ok = true;
        for (uint32_t item = 0;; ++item) {
            const Item& e = item_take(ctl.items, item);
            if (e.steps == 0) break;
            const Segment g = e.segment();
            const int i0 = e.i0 + WtCut::skipped(p, g, e.t), n = e.i1 - e.i0, j = e.t * WT_TILE + row, packed = e.nq * p.group;
            const bool valid = j < e.nk;
            const bool narrow = packed <= 32;           // the first warpgroup has all columns
            // under the triangle: columns of this thread in front of the first row that reads its key, from step i0 on
            const int edge = p.causal && valid ? min(max(j - (g.length - g.nq), 0), g.nq) * p.group - i0 * WT_STEP - 32 * x : 0;
            const bool whole_tile = n == e.steps, mine = x == 0 && valid;
            const float base = mine && whole_tile ? weight_before(sums, e.s, e.h, j) : 0.f;
            f32x2 sum = pack2(0.f, 0.f);
            for (int i = 0; i < n; ++i, ++steps) {
                const uint32_t buffer = steps % WT_BUFFERS;
                ok = ok && mbar_wait(bar(ctl.aux_full[buffer]), (steps / WT_BUFFERS) & 1, abort_word) && mbar_wait(bar(ctl.s_full[buffer]), (steps / WT_BUFFERS) & 1, abort_word);
                ok = __all_sync(~0u, ok);
                tmem_fence_after();
                const int columns = min(packed - (i0 + i) * WT_STEP - 32 * x, 32);
                if (ok && columns > 0) {
                    const int cut = edge - i * WT_STEP;
                    const uint32_t keep = ctl.mask[buffer][x] & (cut <= 0 ? ~0u : cut >= 32 ? 0u : ~0u << cut);
                    const bool whole = __all_sync(~0u, keep == ~0u);
                    const float4* nl = reinterpret_cast<const float4*>(ctl.minus_lse[buffer] + 32 * x);
                    if (columns > 8) {
                        uint32_t v[32];
                        tmem_ld32(S + 128 * buffer, v);
                        tmem_wait_ld(v);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float4 l4 = nl[k];
                            float a, b, c, d;
                            unpack2(fma2(pack2(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1])), sc2, pack2(l4.x, l4.y)), a, b);
                            unpack2(fma2(pack2(__uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3])), sc2, pack2(l4.z, l4.w)), c, d);
                            a = ex2(a);
                            b = ex2(b);
                            c = ex2(c);
                            d = ex2(d);
                            if (!whole) {
                                if (!(keep >> (4 * k) & 1)) a = 0.f;
                                if (!(keep >> (4 * k + 1) & 1)) b = 0.f;
                                if (!(keep >> (4 * k + 2) & 1)) c = 0.f;
                                if (!(keep >> (4 * k + 3) & 1)) d = 0.f;
                            }
                            sum = add2(sum, pack2(a, b));
                            sum = add2(sum, pack2(c, d));
                        }
                    } else {
                        uint32_t v[8];
                        tmem_ld8(S + 128 * buffer, v);
                        tmem_wait_ld(v);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float4 l4 = nl[k];
                            const float l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const float a = ex2(fmaf(__uint_as_float(v[4 * k + c]), scale2, l[c]));
                                if (keep >> (4 * k + c) & 1) sum = add2(sum, pack2(a, 0.f));
                            }
                        }
                    }
                }
                tmem_fence_before();
                mbar_arrive(bar(ctl.s_empty[buffer]));
            }
            float a, b;
            unpack2(sum, a, b);
            float total = a + b;
            if (!narrow) {              // (a buffer is written again two wide items later, behind the meeting of the one in between)
                if (x) ctl.share[wide & 1][x - 1][row] = total;
                asm volatile("bar.sync 1, 512;" ::: "memory");
                if (x == 0)
                    for (int k = 0; k < 3; ++k) total += ctl.share[wide & 1][k][row];
                ++wide;
            }
            if (!(ctl.keys[item % ITEMS][warp % 4] >> lane & 1)) total = 0.f;
            if (!__all_sync(~0u, ok)) total = __int_as_float(0x7fffffff);
            if (mine) {
                if (whole_tile) put_weight(sums, e.s, e.h, j, base + total);
                else w.part[(2LL * blockIdx.x + (e.i0 == 0)) * WT_TILE + row] = total;
            }
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

static size_t weights_carve(const AttnParams& p, void* ws, WtWork* w) {
    Carver cv(ws);
    w->unit_start = cv.take<long long>((size_t)p.n_seg + 1);
    if (counts_itself(p)) w->unit_start = nullptr;
    w->joints = cv.take<Joint>(MAX_SMS);
    w->part = cv.take<float>(2 * (size_t)MAX_SMS * WT_TILE);
    return cv.off;
}

template <typename T, int DP>
static tiga_status launch_weights(AttnParams p, const WtSums& sums, const WtWork& w, cudaStream_t s) {
    TileMaps maps;
    make_tile_maps(&p, operand_type<T>() == 1, &maps);
    const int sms = attention_grid();
    if (sms <= 0) return TIGA_ERR_CUDA;
    TIGA_CUDA_TRY(cudaFuncSetAttribute(attention_weights_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Wt<DP>::SMEM));
    if (w.unit_start) {
        weights_plan_kernel<<<counted(1), PLAN_THREADS, 0, s>>>(p, w.unit_start);
        TIGA_CUDA_TRY(launch_after(attention_weights_kernel<T, DP>, dim3(sms), WT_THREADS, Wt<DP>::SMEM, s, p, sums, w, maps));
    } else attention_weights_kernel<T, DP><<<counted((unsigned)sms), WT_THREADS, Wt<DP>::SMEM, s>>>(p, sums, w, maps);
    TIGA_CUDA_TRY(launch_after(weights_sum_kernel, dim3(sms), WT_TILE, 0, s, p, sums, w));
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
    if (c->max_pages == 0) return TIGA_OK;          // no position
    WtWork w;
    weights_carve(p, ws, &w);
    p.q = q; p.v = p.k; p.q_start = q_start; p.causal = causal != 0; p.lse_in = lse;
    const WtSums sums = {before ? before->data : nullptr, weights->data, before ? before->seg : 0, before ? before->head : 0, weights->seg, weights->head, weights->length};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (h->dtype == TIGA_BF16) return p.D > 64 ? launch_weights<__nv_bfloat16, 128>(p, sums, w, s) : launch_weights<__nv_bfloat16, 64>(p, sums, w, s);
    return p.D > 64 ? launch_weights<__half, 128>(p, sums, w, s) : launch_weights<__half, 64>(p, sums, w, s);
}
