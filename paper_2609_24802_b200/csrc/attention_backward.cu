// Gradients of the online-softmax reducer over dense relations, on the fifth-generation tensor cores.
#include "attention_tiles.cuh"

namespace tiga {

// Two kernels of one form.  A block keeps a stationary tile of 128 rows of two arrays, X1 and X2, and goes through the other side in
// steps of 64 rows of Y1 and Y2:
//     keys and values:  X = (key, value), Y = (q, grad_out):   S = X1 Y1^T, dP = X2 Y2^T (both transposed), grad_value += P Y2,
//                                                               grad_key += dS Y1;      all heads of a group pass by: their sum
//     queries:          X = (q, grad_out), Y = (key, value):   S = X1 Y1^T, dP = X2 Y2^T, grad_q += dS Y1
// with P = exp2(S - lse) and dS = P (dP - delta).  Seven products instead of the five of one kernel that adds grad_q up in memory:
// the sums stay in tensor memory, in one order, so results are reproducible, and no fp32 gradient is written and read again.
// S and dP have two buffers of 64 columns each, so the tensor cores form the next step's while this step's weights are made; P and dS
// lie over them in 16 bits.  Tensor memory: 4 * 64 + 2 * 128 columns, all there is at a width of 128.
// fp16: P carries 2^14 and dS a power of two from the largest norms of the rows of grad_out and value, which bound |dP - delta|: the
// largest value cannot overflow, the smallest keep as many digits as there are.
constexpr int BWD_THREADS = 416, BWD_ROWS = 128, BWD_STEP = 64, BWD_LEAST = 4;
constexpr Geometry KV_GEO = {BWD_ROWS, BWD_STEP, 1}, Q_GEO = {BWD_ROWS, BWD_STEP, 0};

template <int DP> struct Bwd {
    static constexpr int X_TILE = BWD_ROWS * DP * 2, Y_TILE = BWD_STEP * DP * 2;
    static constexpr int STAGES = DP == 128 ? 4 : 8;
    static constexpr int CONTROL = 2 * X_TILE + STAGES * 2 * Y_TILE;
    static constexpr int SMEM = CONTROL + 5120;
};

struct BwdControl {
    unsigned long long full[8], aux_full[8], empty[8], x_full, x_empty, sp_full[2], ps_full[2], acc_full, acc_empty, drain;
    uint32_t tmem, abort_word, never, pad;
    alignas(16) float minus_lse[8][BWD_STEP], minus_delta[8][BWD_STEP];       // keys stationary: of the step's rows
    uint32_t mask[8][4];                                          // queries stationary: the step's keys, 16 bits a producer warp
};
static_assert(sizeof(BwdControl) <= 5120, "control block");

struct BwdWork {
    const long long *kv_start_unit, *q_start_unit;
    float2* stats;                  // [n_q, heads]: lse in log2 (+inf: the row reads nothing), delta
    uint32_t* norms;                // largest squared norms of grad_out and value rows, as bits
    float* part;                    // [2 * grid][rows][sides][DP]
    int kv_rows, q_rows;            // rows that a partial state holds at most
};

// the power of two that dS carries (fp16)
__device__ __forceinline__ float gradient_factor(const uint32_t* norms) {
    const float largest = 2.f * sqrtf(__uint_as_float(norms[0])) * sqrtf(__uint_as_float(norms[1]));
    if (!(largest > 1e-30f && largest < 1e30f)) return 1.f;
    return exp2f(14.f - (float)(ilogbf(largest) + 1));
}

// delta, lse in log2, and the norms behind gradient_factor: 16 lanes a row
constexpr int PREP_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(PREP_THREADS) attention_prepare_kernel(const AttnParams p, const BwdWork w) {
    constexpr bool NORMS = operand_type<T>() == 0;
    const int lane = threadIdx.x % 16;
    const int q_first = clamp_to(p.q_start[0], p.n_q), q_end = max(clamp_to(p.q_start[p.n_seg], p.n_q), q_first);
    const int k_first = clamp_to(p.kv_start[0], p.n_kv), k_end = max(clamp_to(p.kv_start[p.n_seg], p.n_kv), k_first);
    const long long q_rows = (long long)(q_end - q_first) * p.heads, rows = q_rows + (NORMS ? (long long)(k_end - k_first) * p.kv_heads : 0);
    float top_go = 0.f, top_v = 0.f;
    const long long stride = (long long)gridDim.x * (PREP_THREADS / 16);
    for (long long r0 = (long long)blockIdx.x * (PREP_THREADS / 16); r0 < rows; r0 += stride) {      // whole warps stay together
        const long long r = r0 + threadIdx.x / 16;
        float dot = 0.f, norm = 0.f;
        const bool is_q = r < q_rows, on = r < rows && lane * 8 < p.D;
        const long long row = is_q ? q_first + r / p.heads : k_first + (r - q_rows) / p.kv_heads;
        const int head = (int)(is_q ? r % p.heads : (r - q_rows) % p.kv_heads);
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        const T* src = is_q ? (const T*)p.go + row * p.go_row + head * p.go_head : (const T*)p.v + row * p.v_row + head * p.v_head;
        if (on) {
            if (is_q) b = *reinterpret_cast<const uint4*>((const T*)p.o + (row * p.heads + head) * p.D + lane * 8);
            if (is_q || !p.mask || p.mask[row]) a = *reinterpret_cast<const uint4*>(src + lane * 8);
        }
        const T* ea = reinterpret_cast<const T*>(&a);
        const T* eb = reinterpret_cast<const T*>(&b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = Half<T>::to(ea[e]);
            dot += x * Half<T>::to(eb[e]);
            if (NORMS) norm += x * x;
        }
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            dot += __shfl_xor_sync(~0u, dot, d);
            if (NORMS) norm += __shfl_xor_sync(~0u, norm, d);
        }
        if (r >= rows) continue;
        if (is_q) {
            const long long at = row * p.heads + head;
            const float lse = p.lse_in[at];
            const bool reads = lse != -INFINITY;
            if (lane == 0) w.stats[at] = make_float2(reads ? lse * LOG2E_F : INFINITY, reads ? dot : 0.f);
            if (NORMS && reads) top_go = norm == norm ? fmaxf(top_go, norm) : INFINITY;
        } else if (NORMS) top_v = norm == norm ? fmaxf(top_v, norm) : INFINITY;
    }
    if (NORMS) {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            top_go = fmaxf(top_go, __shfl_xor_sync(~0u, top_go, d));
            top_v = fmaxf(top_v, __shfl_xor_sync(~0u, top_v, d));
        }
        if (threadIdx.x % 32 == 0) {        // a maximum does not depend on the order
            atomicMax(&w.norms[0], __float_as_uint(top_go));
            atomicMax(&w.norms[1], __float_as_uint(top_v));
        }
    }
}

template <typename T, int DP, bool KV>
__global__ void __launch_bounds__(BWD_THREADS, 1) attention_backward_kernel(const AttnParams p, const BwdWork w) {
    typedef Bwd<DP> C;
    constexpr Geometry GEO = KV ? KV_GEO : Q_GEO;
    constexpr bool F16 = operand_type<T>() == 0;
    constexpr float BIAS = F16 ? 14.f : 0.f;
    extern __shared__ __align__(1024) unsigned char smem[];
    BwdControl& ctl = *reinterpret_cast<BwdControl*>(smem + C::CONTROL);
    const uint32_t x_tile = smem_u32(smem), ring = x_tile + 2 * C::X_TILE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile uint32_t* abort_word = &ctl.abort_word;
    auto bar = [&](unsigned long long& b) { return smem_u32(&b); };

    const long long* unit_start = KV ? w.kv_start_unit : w.q_start_unit;
    const long long units = unit_start[p.n_seg];
    const long long blocks = blocks_for(units, gridDim.x, BWD_LEAST);
    if (blockIdx.x >= blocks || units == 0) return;
    const long long unit0 = blockIdx.x * units / blocks, unit1 = (blockIdx.x + 1LL) * units / blocks;

    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { mbar_init(bar(ctl.full[i]), 128); mbar_init(bar(ctl.aux_full[i]), 4); mbar_init(bar(ctl.empty[i]), 1); }
        mbar_init(bar(ctl.x_full), 128);
        mbar_init(bar(ctl.x_empty), 1);
        for (int b = 0; b < 2; ++b) { mbar_init(bar(ctl.sp_full[b]), 1); mbar_init(bar(ctl.ps_full[b]), 256); }
        mbar_init(bar(ctl.acc_full), 1);
        mbar_init(bar(ctl.acc_empty), 256);
        mbar_init(bar(ctl.drain), 1);
        ctl.abort_word = ctl.never = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tmem_alloc(smem_u32(&ctl.tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = ctl.tmem;
    const uint32_t s_at[2] = {tmem, tmem + 128}, dp_at[2] = {tmem + 64, tmem + 192}, acc1 = tmem + 256, acc2 = tmem + 384;

    Walker it;
    if (warp >= 8 && warp < 12) {
        // ---------------------------------------------------------------- producers
        const int pw = warp - 8;
        uint32_t steps = 0, items = 0;
        bool ok = true;
        for (bool more = it.begin(p, GEO, unit_start, unit0, unit1); more && ok; more = it.next(p, GEO), ++items) {
            const int packed_rows = it.g.nq * p.group;
            if (items && !(ok = mbar_wait(bar(ctl.x_empty), (items - 1) & 1, abort_word))) break;
            {
                const int r = it.t * BWD_ROWS + 32 * pw + lane;
                long long off1 = -1, off2 = -1;
                if (KV) {
                    const long long j = r < it.g.nk ? key_place(p, it.g, it.s, r) : -1;
                    if (j >= 0) { off1 = j * p.k_row + it.h * p.k_head; off2 = j * p.v_row + it.h * p.v_head; }
                } else if (r < packed_rows) {
                    const PackedRow pr = packed_row(p, it.g, it.h, r);
                    off1 = pr.row * p.q_row + pr.head * p.q_head;
                    off2 = pr.row * p.go_row + pr.head * p.go_head;
                }
                copy_rows<DP, 128, 32>(x_tile, 32 * pw, KV ? p.k : p.q, off1, p.D, unit_start);
                copy_rows<DP, 128, 32>(x_tile + C::X_TILE, 32 * pw, KV ? p.v : p.go, off2, p.D, unit_start);
                cp_async_arrive(bar(ctl.x_full));
            }
            // a step's rows: lane l < 16 has row 16 pw + l
            long long off1, off2;
            float2 stat;
            auto look = [&](int i) {
                const int r = i * BWD_STEP + 16 * pw + lane;
                off1 = off2 = -1;
                stat = make_float2(INFINITY, 0.f);
                if (lane >= 16) return;
                if (KV) {
                    if (r >= packed_rows) return;
                    const PackedRow pr = packed_row(p, it.g, it.h, r);
                    off1 = pr.row * p.q_row + pr.head * p.q_head;
                    off2 = pr.row * p.go_row + pr.head * p.go_head;
                    stat = w.stats[(long long)pr.row * p.heads + pr.head];
                    if (stat.x == INFINITY) off1 = off2 = -1;       // reads nothing: whatever lies there stays out of the products
                } else {
                    const long long j = r < it.g.nk ? key_place(p, it.g, it.s, r) : -1;
                    if (j >= 0) { off1 = j * p.k_row + it.h * p.k_head; off2 = j * p.v_row + it.h * p.v_head; }
                }
            };
            look(it.i0);
            for (int i = it.i0; i < it.i1; ++i, ++steps) {
                const int st = steps % C::STAGES;
                if (steps >= (uint32_t)C::STAGES && !(ok = mbar_wait(bar(ctl.empty[st]), (steps / C::STAGES + 1) & 1, abort_word))) break;
                const long long o1 = off1, o2 = off2;
                if (KV) {
                    if (lane < 16) { ctl.minus_lse[st][16 * pw + lane] = BIAS - stat.x; ctl.minus_delta[st][16 * pw + lane] = -stat.y; }
                } else {
                    const uint32_t valid = __ballot_sync(~0u, off1 >= 0) & 0xffffu;
                    if (lane == 0) ctl.mask[st][pw] = valid;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.aux_full[st]));
                if (i + 1 < it.i1) look(i + 1);
                const uint32_t at = ring + st * 2 * C::Y_TILE;
                copy_rows<DP, BWD_STEP, 16>(at, 16 * pw, KV ? p.q : p.k, o1, p.D, unit_start);
                copy_rows<DP, BWD_STEP, 16>(at + C::Y_TILE, 16 * pw, KV ? p.go : p.v, o2, p.D, unit_start);
                cp_async_arrive(bar(ctl.full[st]));
            }
        }
        cp_async_wait_all();
    } else if (warp == 12) {
        // ---------------------------------------------------------------- matrix instructions
        if (lane == 0) {
            const uint32_t s_shape = mma_shape<T>(BWD_STEP, false), acc_shape = mma_shape<T>(DP, true);
            const uint32_t sign = p.scale < 0.f ? MMA_NEGATE_A : 0;
            uint32_t step0 = 0, items = 0;
            bool ok = true;
            const int pieces = (p.D + 15) / 16;
            auto wait_full = [&](uint32_t step) {
                ok = ok && mbar_wait(bar(ctl.full[step % C::STAGES]), (step / C::STAGES) & 1, abort_word);
                fence_async_proxy();
            };
            auto stage = [&](uint32_t step) { return ring + (step % C::STAGES) * 2 * C::Y_TILE; };
            auto scores = [&](uint32_t step) {
                const uint32_t b = step & 1, y = stage(step);
                for (int k = 0; k < pieces; ++k) {
                    const uint32_t xa = (k / 4) * (BWD_ROWS * 128) + (k % 4) * 32, ya = (k / 4) * (BWD_STEP * 128) + (k % 4) * 32;
                    mma_ss(s_at[b], smem_desc(x_tile + xa, 16), smem_desc(y + ya, 16), s_shape | sign, k > 0);
                }
                for (int k = 0; k < pieces; ++k) {
                    const uint32_t xa = (k / 4) * (BWD_ROWS * 128) + (k % 4) * 32, ya = (k / 4) * (BWD_STEP * 128) + (k % 4) * 32;
                    mma_ss(dp_at[b], smem_desc(x_tile + C::X_TILE + xa, 16), smem_desc(y + C::Y_TILE + ya, 16), s_shape, k > 0);
                }
                mma_commit(bar(ctl.sp_full[b]));
            };
            for (bool more = it.begin(p, GEO, unit_start, unit0, unit1); more && ok; more = it.next(p, GEO), ++items) {
                const int n = it.i1 - it.i0;
                ok = ok && mbar_wait(bar(ctl.x_full), items & 1, abort_word);
                wait_full(step0);
                if (!ok) break;
                scores(step0);
                if (n == 1) mma_commit(bar(ctl.x_empty));
                for (int i = 0; i < n; ++i) {
                    const uint32_t step = step0 + i, b = step & 1;
                    if (i + 1 < n) {
                        wait_full(step + 1);
                        if (!ok) break;
                        scores(step + 1);
                        if (i + 2 == n) mma_commit(bar(ctl.x_empty));
                    }
                    if (i == 0 && items) ok = ok && mbar_wait(bar(ctl.acc_empty), (items - 1) & 1, abort_word);
                    ok = ok && mbar_wait(bar(ctl.ps_full[b]), (step / 2) & 1, abort_word);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t y = stage(step);
#pragma unroll
                    for (int k = 0; k < BWD_STEP / 16; ++k) {
                        const uint32_t a = (k / 2) * 32 + (k % 2) * 8;
                        if (KV) mma_ts(acc2, s_at[b] + a, smem_desc(y + C::Y_TILE + k * 2048, BWD_STEP * 128), acc_shape, i > 0 || k > 0);
                        mma_ts(acc1, dp_at[b] + a, smem_desc(y + k * 2048, BWD_STEP * 128), acc_shape, i > 0 || k > 0);
                    }
                    mma_commit(bar(ctl.empty[step % C::STAGES]));
                }
                if (!ok) break;
                mma_commit(bar(ctl.acc_full));
                step0 += n;
            }
            mma_commit(bar(ctl.drain));
            mbar_wait(bar(ctl.drain), 0, &ctl.never);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- weights: warpgroup x has 32 of a step's 64 columns
        const int x = warp / 4;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const int row = threadIdx.x & 127;
        const float scale2 = fmaxf(fabsf(p.scale) * LOG2E_F, 1e-30f);
        const float factor = F16 ? gradient_factor(w.norms) : 1.f;
        const f32x2 sc2 = dup2(scale2), ds2 = dup2(F16 ? factor * 0x1p-14f : 1.f);
        uint32_t step0 = 0, items = 0;
        bool ok = true;
        for (bool more = it.begin(p, GEO, unit_start, unit0, unit1); more; more = it.next(p, GEO), ++items) {
            const int n = it.i1 - it.i0, r = it.t * BWD_ROWS + row;
            const bool valid = r < stationary_rows(p, it.g, GEO);
            const bool warp_on = (r & ~31) < stationary_rows(p, it.g, GEO);
            f32x2 my_lse = 0, my_delta = 0;
            long long out_row = 0;
            bool masked = false;
            if (KV) {
                out_row = (long long)(it.g.k0 + r) * p.kv_heads + it.h;
                masked = valid && key_place(p, it.g, it.s, r) < 0;
            } else if (valid) {
                const PackedRow pr = packed_row(p, it.g, it.h, r);
                out_row = (long long)pr.row * p.heads + pr.head;
                const float2 st = w.stats[out_row];
                my_lse = dup2(BIAS - st.x);
                my_delta = dup2(-st.y);
                masked = st.x == INFINITY;
            }
            for (int i = 0; i < n; ++i) {
                const uint32_t step = step0 + i, b = step & 1, st = step % C::STAGES;
                ok = ok && mbar_wait(bar(ctl.aux_full[st]), (step / C::STAGES) & 1, abort_word) && mbar_wait(bar(ctl.sp_full[b]), (step / 2) & 1, abort_word);
                ok = __all_sync(~0u, ok);
                if (!ok) continue;
                tmem_fence_after();
                if (warp_on) {
                    uint32_t s[32], d[32];
                    tmem_ld32(s_at[b] + lanes + 32 * x, s);
                    tmem_ld32(dp_at[b] + lanes + 32 * x, d);
                    uint32_t keep = ~0u;
                    if (!KV) keep = ctl.mask[st][2 * x] | ctl.mask[st][2 * x + 1] << 16;
                    tmem_wait_ld();
                    uint32_t pk[16], dk[16];
                    const float4* nl = reinterpret_cast<const float4*>(ctl.minus_lse[st] + 32 * x);
                    const float4* nd = reinterpret_cast<const float4*>(ctl.minus_delta[st] + 32 * x);
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        float4 l4, d4;
                        if (KV) { l4 = nl[k / 2]; d4 = nd[k / 2]; }
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const f32x2 lse = KV ? (e ? pack2(l4.z, l4.w) : pack2(l4.x, l4.y)) : my_lse;
                            const f32x2 delta = KV ? (e ? pack2(d4.z, d4.w) : pack2(d4.x, d4.y)) : my_delta;
                            const int c = 2 * (k + e);
                            float a0, a1, g0, g1;
                            unpack2(fma2(pack2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sc2, lse), a0, a1);
                            a0 = ex2(a0);
                            a1 = ex2(a1);
                            if (!KV && keep != ~0u) {
                                if (!(keep >> c & 1)) a0 = 0.f;
                                if (!(keep >> (c + 1) & 1)) a1 = 0.f;
                            }
                            if (KV) pk[k + e] = pack_half<T>(a0, a1);
                            f32x2 g = mul2(pack2(a0, a1), add2(pack2(__uint_as_float(d[c]), __uint_as_float(d[c + 1])), delta));
                            if (F16) g = mul2(g, ds2);
                            unpack2(g, g0, g1);
                            dk[k + e] = pack_half<T>(g0, g1);
                        }
                    }
                    if (KV) tmem_st16(s_at[b] + lanes + 32 * x, pk);
                    tmem_st16(dp_at[b] + lanes + 32 * x, dk);
                    tmem_wait_st();
                }
                tmem_fence_before();
                mbar_arrive(bar(ctl.ps_full[b]));
            }
            ok = ok && mbar_wait(bar(ctl.acc_full), items & 1, abort_word);
            ok = __all_sync(~0u, ok);
            tmem_fence_after();
            // keys stationary: warpgroup 0 writes grad_key, 1 grad_value; queries: a half of grad_q's features each
            const bool whole_tile = it.i0 == 0 && it.i1 == it.steps;
            const int rows = KV ? w.kv_rows : w.q_rows;
            constexpr int SIDES = KV ? 2 : 1;
            const uint32_t acc = KV && x ? acc2 : acc1;
            const float finish = KV && x ? (F16 ? 0x1p-14f : 1.f) : p.scale / factor;
            T* out = (T*)(KV ? (x ? p.gv : p.gk) : p.gq);
            float* part = w.part + ((((2LL * blockIdx.x + (it.i0 == 0)) * rows + row) * SIDES) + (KV ? x : 0)) * DP;
            const int c0 = KV ? 0 : x * (DP / 64), c1 = KV ? DP / 32 : c0 + DP / 64;
            if (warp_on)
                for (int c = c0; c < c1; ++c) {
                    uint32_t v[32];
                    tmem_ld32(acc + lanes + 32 * c, v);
                    tmem_wait_ld();
                    if (!valid) continue;
                    if (!ok)
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = 0x7fffffffu;
                    if (whole_tile) {
                        if (!out) continue;
                        uint4* o4 = reinterpret_cast<uint4*>(out + out_row * p.D + 32 * c);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if (32 * c + 8 * k >= p.D) continue;
                            uint32_t o[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                o[e] = masked && ok ? 0u : pack_half<T>(__uint_as_float(v[8 * k + 2 * e]) * finish, __uint_as_float(v[8 * k + 2 * e + 1]) * finish);
                            o4[k] = make_uint4(o[0], o[1], o[2], o[3]);
                        }
                    } else {
                        uint4* o4 = reinterpret_cast<uint4*>(part + 32 * c);
#pragma unroll
                        for (int k = 0; k < 8; ++k) o4[k] = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                    }
                }
            tmem_fence_before();
            mbar_arrive(bar(ctl.acc_empty));
            step0 += n;
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 12) { tmem_fence_after(); tmem_free(tmem, 512); }
}

// Adds up the partial sums of a tile that several blocks shared, in the order of its steps.  A warp has a row of one gradient; many parts
// (few tiles, a long axis) are shared by the block's warps, whose sums are added in order.
constexpr int SUM_WARPS = 8, SUM_Y = 16, SUM_FEW = 8;

template <typename T, int DP, bool KV>
__global__ void __launch_bounds__(SUM_WARPS * 32) attention_sum_kernel(const AttnParams p, const BwdWork w) {
    constexpr Geometry GEO = KV ? KV_GEO : Q_GEO;
    constexpr int SIDES = KV ? 2 : 1, E = DP / 32;
    constexpr bool F16 = operand_type<T>() == 0;
    const long long* unit_start = KV ? w.kv_start_unit : w.q_start_unit;
    const long long units = unit_start[p.n_seg];
    const long long blocks = blocks_for(units, gridDim.x, BWD_LEAST);
    if (blockIdx.x >= blocks || units == 0) return;
    const long long unit0 = blockIdx.x * units / blocks, unit1 = (blockIdx.x + 1LL) * units / blocks;
    Walker it;
    if (!it.begin(p, GEO, unit_start, unit0, unit1) || it.i0 == 0 || it.i1 < it.steps) return;
    const int first = (int)(((unit0 - it.i0 + 1) * blocks - 1) / units);        // the block in which the tile begins
    const int parts = (int)blockIdx.x - first + 1;
    const int rows = min(stationary_rows(p, it.g, GEO) - it.t * BWD_ROWS, BWD_ROWS), cap = KV ? w.kv_rows : w.q_rows;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const float factor = F16 ? gradient_factor(w.norms) : 1.f;
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
            const float* src = w.part + (((2LL * (first + k) + (k == 0)) * cap + r) * SIDES + side) * DP;
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
            if (KV) {
                out_row = (long long)(it.g.k0 + n) * p.kv_heads + it.h;
                masked = key_place(p, it.g, it.s, n) < 0;
            } else {
                const PackedRow pr = packed_row(p, it.g, it.h, n);
                out_row = (long long)pr.row * p.heads + pr.head;
                masked = w.stats[out_row].x == INFINITY;
            }
            const float finish = KV && side ? (F16 ? 0x1p-14f : 1.f) : p.scale / factor;
            T* out = (T*)(KV ? (side ? p.gv : p.gk) : p.gq);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (out && lane + 32 * e < p.D) out[out_row * p.D + lane + 32 * e] = Half<T>::from(masked ? 0.f : o[e] * finish);
        }
    }
}

static __global__ void __launch_bounds__(PLAN_THREADS) backward_plan_kernel(const AttnParams p, long long* kv_units, long long* q_units, uint32_t* norms) {
    if (blockIdx.x == 0) {
        if (threadIdx.x < 2) norms[threadIdx.x] = 0;
        plan_units(p, KV_GEO, kv_units);
    } else plan_units(p, Q_GEO, q_units);
}

static size_t backward_carve(const AttnParams& p, void* ws, BwdWork* w) {
    const size_t slots = 2 * (size_t)MAX_SMS, dp = p.D > 64 ? 128 : 64;
    const long long packed = (long long)p.n_q * p.group;
    w->kv_rows = p.n_kv < BWD_ROWS ? p.n_kv : BWD_ROWS;
    w->q_rows = (int)(packed < BWD_ROWS ? packed : BWD_ROWS);
    const size_t floats = (size_t)w->kv_rows * 2 > (size_t)w->q_rows ? (size_t)w->kv_rows * 2 : (size_t)w->q_rows;
    Carver cv(ws);
    w->kv_start_unit = cv.take<long long>((size_t)p.n_seg + 1);
    w->q_start_unit = cv.take<long long>((size_t)p.n_seg + 1);
    w->norms = cv.take<uint32_t>(2);
    w->stats = cv.take<float2>((size_t)p.n_q * p.heads);
    w->part = cv.take<float>(slots * floats * dp);          // the key kernel's, then the query kernel's
    return cv.off;
}
size_t attention_backward_bytes(const AttnParams& p) { BwdWork w; return backward_carve(p, nullptr, &w); }

template <typename T, int DP, bool KV>
static tiga_status launch_side(const AttnParams& p, const BwdWork& w, int sms, cudaStream_t s) {
    TIGA_CUDA_TRY(cudaFuncSetAttribute(attention_backward_kernel<T, DP, KV>, cudaFuncAttributeMaxDynamicSharedMemorySize, Bwd<DP>::SMEM));
    attention_backward_kernel<T, DP, KV><<<counted((unsigned)sms), BWD_THREADS, Bwd<DP>::SMEM, s>>>(p, w);
    attention_sum_kernel<T, DP, KV><<<counted(dim3(sms, SUM_Y)), SUM_WARPS * 32, 0, s>>>(p, w);
    return launch_status();
}

template <typename T, int DP>
static tiga_status launch_backward(const AttnParams& p, const BwdWork& w, cudaStream_t s) {
    const int sms = attention_grid();
    if (sms <= 0) return TIGA_ERR_CUDA;
    backward_plan_kernel<<<counted(2), PLAN_THREADS, 0, s>>>(p, const_cast<long long*>(w.kv_start_unit), const_cast<long long*>(w.q_start_unit), w.norms);
    const long long rows = (long long)p.n_q * p.heads + (long long)p.n_kv * p.kv_heads;
    const long long grid = (rows * 16 + PREP_THREADS - 1) / PREP_THREADS;
    attention_prepare_kernel<T><<<counted((unsigned)(grid < 8 * sms ? grid : 8 * sms)), PREP_THREADS, 0, s>>>(p, w);
    tiga_status st = launch_status();
    if (st == TIGA_OK && (p.gk || p.gv) && p.n_kv) st = launch_side<T, DP, true>(p, w, sms, s);
    if (st == TIGA_OK && p.gq && p.n_q) st = launch_side<T, DP, false>(p, w, sms, s);
    return st;
}

tiga_status attention_backward(const AttnParams& p, bool bf16, void* ws, cudaStream_t s) {
    BwdWork w;
    backward_carve(p, ws, &w);
    if (bf16) return p.D > 64 ? launch_backward<__nv_bfloat16, 128>(p, w, s) : launch_backward<__nv_bfloat16, 64>(p, w, s);
    return p.D > 64 ? launch_backward<__half, 128>(p, w, s) : launch_backward<__half, 64>(p, w, s);
}

}  // namespace tiga
