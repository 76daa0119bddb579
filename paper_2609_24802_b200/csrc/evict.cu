// A paged cache is cut to a budget: every kv head of a sequence keeps its last positions and those that carry the most weight.
#include <algorithm>
#include <cooperative_groups.h>
#include "attention_shared.cuh"

namespace tiga {

// ---- Which positions stay.  A list is the positions of one (sequence, kv head).  Weights become whole numbers of the same order (rank_of),
// above all of them the last positions, below all of them those that have no page: the `keep` largest stay, of equal ones the first, and
// come out in the order of their positions.
// The keep-th largest is found digit by digit (11 + 11 + 10 bits): counts of a digit among the numbers that agree with the digits found so
// far, added up from the top.  Then every warp, whose positions follow one another, knows from the warps in front how many it puts where.
// A list has one block, or a cluster of SELECT_CLUSTER that share its positions and read one another's counts.  What bounds it: many lists, the
// instructions of five passes over numbers in shared memory; few lists, the steps one after the other.  So many lists have small blocks, of which
// an SM holds several (512 lists of up to 8192: 46 us with 1024 threads each, 34 with 256).
constexpr int SELECT_MANY = 256, SELECT_FEW = 1024, SELECT_BINS = 2048, SELECT_CLUSTER = 8;            // threads
constexpr int SELECT_AT_ONCE = 8;               // positions that a lane loads together
constexpr int SELECT_HELD = 40960;              // numbers that a block's shared memory holds

struct EvictParams {
    const float* weights;
    float* to_weights;              // NULL: not wanted
    const int32_t *table, *kv_len, *to_table;
    int32_t *kept, *to_len;
    const char *key, *value;
    char *to_key, *to_value;
    long long w_seg, w_head, w_length, o_seg, o_head, o_length;
    long long n_pages, page_size, max_pages, table_stride, page_stride, slot_stride, head_stride;           // strides in bytes from here on
    long long to_pages, to_page_size, to_max_pages, to_table_stride, to_page_stride, to_slot_stride, to_head_stride;
    int n_seg, kv_heads, pieces;    // pieces of 16 bytes of a row
    long long keep, recent;
    int held;                       // numbers that shared memory holds in this launch
};

__device__ __forceinline__ int page_of(const int32_t* table, long long stride, int s, long long page, long long n_pages) {
    const int id = table[s * stride + page];
    return id >= 0 && id < n_pages ? id : -1;
}

// order of the weights as unsigned numbers: 0 is no position at all, NaN comes in front of -inf, -0 equals 0
__device__ __forceinline__ uint32_t rank_of(float w) {
    if (w != w) return 1;
    if (w == 0.f) return 0x80000000u;
    const uint32_t b = __float_as_uint(w);
    return b >> 31 ? ~b : b | 0x80000000u;
}
constexpr uint32_t LAST_POSITION = 0xffffffffu;

// Keys and values of 32 places of a list, from `place` on, by a warp, 16 bytes a lane: a lane looks up where one of them comes from and goes to,
// then the lanes of a row copy it together.  Bound by memory: what stays is read and written once.
template <typename F>
__device__ __forceinline__ void move_places(const EvictParams& p, const long long list, const long long first, F wait_for_kept) {
    const int lane = threadIdx.x % 32, s = (int)quotient(list, p.kv_heads), h = (int)(list - (long long)s * p.kv_heads);
    const long long place = first + lane;
    long long to = -1, from = -1;
    if (place < p.keep) {                   // (the target's page does not depend on what stays)
        const long long page = quotient(place, p.to_page_size);
        const int id = page < p.to_max_pages ? page_of(p.to_table, p.to_table_stride, s, page, p.to_pages) : -1;
        if (id >= 0) to = id * p.to_page_stride + (place - page * p.to_page_size) * p.to_slot_stride + h * p.to_head_stride;
    }
    wait_for_kept();
    if (to >= 0) {
        const int j = p.kept[list * p.keep + place];
        if (j >= 0) {
            const long long page = quotient(j, p.page_size);
            const int id = page_of(p.table, p.table_stride, s, page, p.n_pages);
            if (id >= 0) from = id * p.page_stride + (j - page * p.page_size) * p.slot_stride + h * p.head_stride;
        }
    }
    const int rows = 32 / p.pieces, row = lane / p.pieces, piece = lane - row * p.pieces;           // rows at once; the lanes behind them are idle
    for (int r0 = 0; r0 < 32; r0 += 4 * rows) {
        uint4 k[4], v[4];
        long long a[4], b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + u * rows + row;
            a[u] = __shfl_sync(~0u, from, r & 31);
            b[u] = __shfl_sync(~0u, to, r & 31);
            if (r >= 32 || row >= rows) a[u] = -1;
            if (a[u] >= 0) {
                k[u] = __ldcs(reinterpret_cast<const uint4*>(p.key + a[u]) + piece);
                v[u] = __ldcs(reinterpret_cast<const uint4*>(p.value + a[u]) + piece);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (a[u] >= 0) {
                reinterpret_cast<uint4*>(p.to_key + b[u])[piece] = k[u];
                reinterpret_cast<uint4*>(p.to_value + b[u])[piece] = v[u];
            }
    }
}

template <int THREADS, int CLUSTER, bool MOVE>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_select_kernel(const EvictParams p) {
    namespace cg = cooperative_groups;
    constexpr int WARPS = THREADS / 32;
    extern __shared__ uint32_t numbers[];
    __shared__ uint32_t bins[SELECT_BINS], warp_sum[32], found[2];              // found: digit, how many more of it are wanted
    __shared__ uint32_t above[32], equal[32], totals[4];                        // totals: positions there are, above, equal (of this block)
    let_next_kernel_start();
    const int list = blockIdx.x / CLUSTER, part = blockIdx.x % CLUSTER, s = list / p.kv_heads, h = list % p.kv_heads;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int length = max(p.kv_len[s], 0), n = (int)min(min((long long)length, p.max_pages * p.page_size), MOST_ROWS);
    const int recent = (int)max((long long)length - p.recent, 0LL), weighed = (int)min((long long)n, p.w_length);         // the last positions begin, the weights end
    // this block's positions, and the warp's (whole groups of 32)
    const int per_warp = ((n + CLUSTER * WARPS - 1) / (CLUSTER * WARPS) + 31) / 32 * 32;
    const int begin = (int)min((long long)per_warp * WARPS * part, (long long)n), end = (int)min((long long)begin + per_warp * WARPS, (long long)n);
    const int w0 = (int)min((long long)begin + (long long)per_warp * warp, (long long)end), w1 = (int)min((long long)w0 + per_warp, (long long)end);
    const bool held = end - begin <= p.held;
    const float* weights = p.weights + s * p.w_seg + h * p.w_head;
    const uint32_t page_size = (uint32_t)p.page_size;
    const int32_t* table = p.table + s * p.table_stride;
    auto weight_of = [&](int j) { return j < min(weighed, w1) ? __ldg(weights + j) : 0.f; };
    auto id_of = [&](int j, uint32_t page) { return j < w1 ? __ldg(table + page) : -1; };
    auto number_of = [&](int j, float w, int id) -> uint32_t { return id < 0 || id >= p.n_pages ? 0 : j >= recent ? LAST_POSITION : rank_of(w); };
    auto number = [&](int j) { return held ? numbers[j - begin] : number_of(j, weight_of(j), id_of(j, (uint32_t)j / page_size)); };
    auto meet = [&]() { if (CLUSTER > 1) cg::this_cluster().sync(); else __syncthreads(); };
    auto of_block = [&](uint32_t* a, int b) { return CLUSTER > 1 ? cg::this_cluster().map_shared_rank(a, b) : a; };

    // ---- the numbers, how many positions there are, and the counts of the first digit (the last positions' apart: a crowd in one bin)
    for (int k = threadIdx.x; k < SELECT_BINS; k += THREADS) bins[k] = 0;
    __syncthreads();
    uint32_t there = 0, last = 0;
    // (a lane's loads stand in front of its stores, for which they would wait: these lists 44 us instead of 36, the pass at the end included)
    const uint32_t pages_on = 32 / page_size, slots_on = 32 % page_size;            // 32 positions on (with a division for each 2 us more)
    uint32_t page = (uint32_t)(w0 + lane) / page_size, slot = (uint32_t)(w0 + lane) % page_size;
    for (int j0 = w0; j0 < w1; j0 += 32 * SELECT_AT_ONCE) {
        float w[SELECT_AT_ONCE];
        int id[SELECT_AT_ONCE];
#pragma unroll
        for (int u = 0; u < SELECT_AT_ONCE; ++u) {
            const int j = j0 + 32 * u + lane;
            w[u] = weight_of(j);
            id[u] = id_of(j, page);
            page += pages_on;
            slot += slots_on;
            if (slot >= page_size) { slot -= page_size; ++page; }
        }
#pragma unroll
        for (int u = 0; u < SELECT_AT_ONCE; ++u) {
            const int j = j0 + 32 * u + lane;
            if (j >= w1) break;
            const uint32_t v = number_of(j, w[u], id[u]);
            if (held) numbers[j - begin] = v;
            there += v != 0;
            if (v == LAST_POSITION) ++last;
            else if (v) atomicAdd(&bins[v >> 21], 1u);
        }
    }
    there = __reduce_add_sync(~0u, there);
    last = __reduce_add_sync(~0u, last);
    if (lane == 0) {
        warp_sum[warp] = there;
        if (last) atomicAdd(&bins[LAST_POSITION >> 21], last);
    }
    __syncthreads();
    if (warp == 0) {
        const uint32_t sum = __reduce_add_sync(~0u, lane < WARPS ? warp_sum[lane] : 0u);
        if (lane == 0) totals[0] = sum;
    }
    meet();
    uint32_t all = 0;
    for (int b = 0; b < CLUSTER; ++b) all += of_block(totals, b)[0];
    const uint32_t stay = (uint32_t)min((long long)all, p.keep);

    // ---- the smallest number that stays, and how many of those equal to it
    uint32_t border = 0, wanted = 0;            // 0: everything that there is stays
    if (all > stay) {
        wanted = stay;
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, size = digit < 2 ? 2048 : 1024;
            if (digit) {
                const uint32_t high = ~0u << (digit == 1 ? 21 : 10);            // the digits that are found
                for (int k = threadIdx.x; k < size; k += THREADS) bins[k] = 0;
                __syncthreads();
                if (border == (LAST_POSITION & high)) {         // (the last positions may be most of these)
                    last = 0;
                    for (int j = w0 + lane; j < w1; j += 32) {
                        const uint32_t v = number(j);
                        if (v == LAST_POSITION) ++last;
                        else if ((v & high) == border) atomicAdd(&bins[v >> shift & (size - 1)], 1u);
                    }
                    last = __reduce_add_sync(~0u, last);
                    if (lane == 0 && last) atomicAdd(&bins[size - 1], last);
                } else
#pragma unroll 4
                    for (int j = w0 + lane; j < w1; j += 32) {
                        const uint32_t v = number(j);
                        if ((v & high) == border && v) atomicAdd(&bins[v >> shift & (size - 1)], 1u);
                    }
                meet();
            }
            // thread k has `per` bins, counted from the top
            const int per = size / THREADS > 0 ? size / THREADS : 1, top = size - 1 - per * (int)threadIdx.x;
            uint32_t mine = 0, run;
            if (top >= 0)
                for (int b = 0; b < CLUSTER; ++b) { const uint32_t* o = of_block(bins, b); for (int k = 0; k < per; ++k) mine += o[top - k]; }
            run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(~0u, run, o); if (lane >= o) run += u; }
            if (lane == 31) warp_sum[warp] = run;
            __syncthreads();
            const uint32_t in_front = lane < warp ? warp_sum[lane] : 0u;
            uint32_t before = run - mine + __reduce_add_sync(~0u, in_front);
            if (before < wanted && wanted <= before + mine) {           // one thread
                for (int k = 0; k < per; ++k) {
                    uint32_t count = 0;
                    for (int b = 0; b < CLUSTER; ++b) count += of_block(bins, b)[top - k];
                    if (wanted <= before + count) { found[0] = top - k; found[1] = wanted - before; break; }
                    before += count;
                }
            }
            meet();             // (nobody clears its bins while they are read)
            border |= found[0] << shift;
            wanted = found[1];
        }
    }

    // ---- where they go: numbers above the border and the first ones equal to it, in the order of their positions
    uint32_t n_above = 0, n_equal = 0;
#pragma unroll 4
    for (int j = w0 + lane; j < w1; j += 32) {
        const uint32_t v = number(j);
        n_above += v > border;
        n_equal += v == border && v != 0;
    }
    n_above = __reduce_add_sync(~0u, n_above);
    n_equal = __reduce_add_sync(~0u, n_equal);
    if (lane == 0) { above[warp] = n_above; equal[warp] = n_equal; }
    __syncthreads();
    const uint32_t above_in_front = lane < warp ? above[lane] : 0u, equal_in_front = lane < warp ? equal[lane] : 0u;
    uint32_t ahead_above = __reduce_add_sync(~0u, above_in_front), ahead_equal = __reduce_add_sync(~0u, equal_in_front);
    if (CLUSTER > 1) {
        if (warp == WARPS - 1 && lane == 0) { totals[1] = ahead_above + n_above; totals[2] = ahead_equal + n_equal; }
        meet();
        for (int b = 0; b < part; ++b) { ahead_above += of_block(totals, b)[1]; ahead_equal += of_block(totals, b)[2]; }
        meet();                 // (a block's shared memory is there until the last one has read it)
    }
    int32_t* kept = p.kept + (long long)list * p.keep;
    float* to = p.to_weights ? p.to_weights + s * p.o_seg + h * p.o_head : nullptr;
    for (int j0 = w0; j0 < w1; j0 += 32 * SELECT_AT_ONCE) {
        float w[SELECT_AT_ONCE];
        if (to)
#pragma unroll
            for (int u = 0; u < SELECT_AT_ONCE; ++u) w[u] = weight_of(j0 + 32 * u + lane);
#pragma unroll
        for (int u = 0; u < SELECT_AT_ONCE; ++u) {
            const int j = j0 + 32 * u + lane;
            const uint32_t v = j < w1 ? number(j) : 0;
            const uint32_t over = __ballot_sync(~0u, v > border), same = __ballot_sync(~0u, v == border && v != 0), behind = (1u << lane) - 1;
            const uint32_t before_equal = ahead_equal + __popc(same & behind);
            const uint32_t at = ahead_above + __popc(over & behind) + min(before_equal, wanted);
            if (v > border || (v == border && v != 0 && before_equal < wanted)) {
                kept[at] = j;
                if (to && at < p.o_length) to[at] = w[u];
            }
            ahead_above += __popc(over);
            ahead_equal += __popc(same);
        }
    }
    const long long thread = (long long)part * THREADS + threadIdx.x;
    for (long long k = stay + thread; k < p.keep; k += CLUSTER * THREADS) kept[k] = -1;
    if (to) for (long long k = stay + thread; k < p.o_length; k += CLUSTER * THREADS) to[k] = 0.f;
    if (h == 0 && thread == 0) p.to_len[s] = (int32_t)stay;
    if (MOVE) {
        __syncthreads();
        for (long long place = 32 * warp; place < stay; place += THREADS) move_places(p, list, place, [] {});
    }
}

// ---- Few short lists are moved by the block that selects (a launch less: 5 us of the host), others by a kernel with a warp for 32 places.
constexpr int MOVE_THREADS = 256;
__global__ void __launch_bounds__(MOVE_THREADS) evict_move_kernel(const EvictParams p, const long long tasks) {
    const long long task = (long long)blockIdx.x * (MOVE_THREADS / 32) + threadIdx.x / 32;
    if (task >= tasks) return;
    const long long per_list = quotient(p.keep + 31, 32), list = quotient(task, per_list);
    move_places(p, list, (task - list * per_list) * 32, [] { wait_for_previous_kernel(); });
}

template <int THREADS, int CLUSTER, bool MOVE>
static cudaError_t launch_select(EvictParams p, long long most, long long lists, cudaStream_t s) {
    // a block's part of the longest list, as it is cut there
    const long long share = (most + CLUSTER * THREADS - 1) / (CLUSTER * THREADS) * THREADS;
    p.held = (int)(share < SELECT_HELD ? share : SELECT_HELD);
    const size_t smem = (size_t)p.held * 4;
    if (smem > 32 * 1024) {         // (beside the counts; more than any kernel may have unasked)
        const cudaError_t e = cudaFuncSetAttribute(evict_select_kernel<THREADS, CLUSTER, MOVE>, cudaFuncAttributeMaxDynamicSharedMemorySize, SELECT_HELD * 4);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)(lists * CLUSTER));
    c.blockDim = dim3(THREADS);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute a{};
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = CLUSTER;
    a.val.clusterDim.y = a.val.clusterDim.z = 1;
    c.attrs = &a;
    c.numAttrs = CLUSTER > 1;
    note_launch();
    return cudaLaunchKernelEx(&c, evict_select_kernel<THREADS, CLUSTER, MOVE>, p);
}

// Whether rows (of a page, slot and head) lie in one another, so that two warps would write the same place: of the three strides each has to
// be as long as what the shorter ones span.
static bool rows_share_storage(const tiga_pages* c, int kv_heads, int D) {
    struct Axis { long long stride, n; } axes[3] = {{c->page_stride, c->n_pages}, {c->slot_stride, c->page_size}, {c->head_stride, kv_heads}};
    std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
    __int128 span = D;
    for (const Axis& a : axes) {
        if (a.n < 2) continue;
        if (a.stride < span) return true;
        span += (__int128)a.stride * (a.n - 1);
    }
    return false;
}

}  // namespace tiga

using namespace tiga;

extern "C" tiga_status tiga_paged_evict(const tiga_pages* from, const tiga_pages* to, const tiga_heads* h, const tiga_weights* weights,
                                        int64_t keep, int64_t recent, const tiga_weights* to_weights, int32_t* to_len, int32_t* kept, void* stream) {
    tiga_status st = attention_heads_check(h);
    if (st != TIGA_OK) return st;
    if ((st = attention_pages_check(from)) != TIGA_OK || (st = attention_pages_check(to)) != TIGA_OK) return st;
    if (from->n_seg != to->n_seg || keep < 1 || recent < 0 || recent > keep) return TIGA_ERR_INVALID_ARG;
    if (to->page_size * to->max_pages < keep) return TIGA_ERR_INVALID_ARG;              // the budget needs that many places
    if (attention_bad_weights(weights) || (to_weights && attention_bad_weights(to_weights))) return TIGA_ERR_INVALID_ARG;
    if (keep > MOST_ROWS || from->n_seg * h->kv_heads > (1 << 24)) return TIGA_ERR_UNSUPPORTED;
    if (from->n_seg == 0) return TIGA_OK;
    if (rows_share_storage(to, h->kv_heads, h->D)) return TIGA_ERR_INVALID_ARG;
    if (attention_bad_ints(from->kv_len) || attention_bad_ints(to_len) || attention_bad_ints(kept) || to_len == from->kv_len) return TIGA_ERR_INVALID_ARG;
    if (attention_bad_ints(to->table) || (from->max_pages > 0 && attention_bad_ints(from->table))) return TIGA_ERR_INVALID_ARG;
    auto bad = [](const void* a) { return !a || !aligned16(a); };
    if ((from->n_pages > 0 && (bad(from->key) || bad(from->value))) || (to->n_pages > 0 && (bad(to->key) || bad(to->value)))) return TIGA_ERR_INVALID_ARG;
    if ((weights->length > 0 && bad(weights->data)) || (to_weights && to_weights->length > 0 && bad(to_weights->data))) return TIGA_ERR_INVALID_ARG;
    if (to_weights && (attention_weights_overlap(to_weights, from->n_seg, h->kv_heads) || (to_weights->length > 0 && to_weights->data == weights->data))) return TIGA_ERR_INVALID_ARG;

    EvictParams p{};
    p.weights = weights->data; p.w_seg = weights->seg; p.w_head = weights->head; p.w_length = weights->length;
    if (to_weights) { p.to_weights = to_weights->data; p.o_seg = to_weights->seg; p.o_head = to_weights->head; p.o_length = to_weights->length; }
    p.table = from->table; p.kv_len = from->kv_len; p.to_table = to->table; p.kept = kept; p.to_len = to_len;
    p.key = (const char*)from->key; p.value = (const char*)from->value; p.to_key = (char*)to->key; p.to_value = (char*)to->value;
    p.n_pages = from->n_pages; p.page_size = from->page_size; p.max_pages = from->max_pages; p.table_stride = from->table_stride;
    p.page_stride = 2 * from->page_stride; p.slot_stride = 2 * from->slot_stride; p.head_stride = 2 * from->head_stride;
    p.to_pages = to->n_pages; p.to_page_size = to->page_size; p.to_max_pages = to->max_pages; p.to_table_stride = to->table_stride;
    p.to_page_stride = 2 * to->page_stride; p.to_slot_stride = 2 * to->slot_stride; p.to_head_stride = 2 * to->head_stride;
    p.n_seg = (int)from->n_seg; p.kv_heads = h->kv_heads; p.pieces = h->D / 8;
    p.keep = keep; p.recent = recent;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long lists = (long long)p.n_seg * p.kv_heads, most = p.max_pages * p.page_size;
    int dev = 0, sms = 0;
    TIGA_CUDA_TRY(cudaGetDevice(&dev));
    TIGA_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // Up to 512 places of few short lists are moved by the block that selects them: 2 to 4 us more on the device for 5 us of the host's launch (2 lists
    // of 8192, 512 kept: 22.7 against 18.6; 1024 kept: 27.6 against 18.6; behind longer lists the launch does not show).
    // A cluster for each list where one block's shared memory does not hold it and the lists alone leave most SMs idle: a list's meetings cost 15 us, and
    // no more than about 16 clusters find room at once (16 lists of 40960: 59 us, a block each 40; of 45056: 60 and 99; 64 lists of 57344: 145 and 121).
    // Small blocks where there are several for each SM, whose shared memory holds their numbers (2048 lists of 8192: 97 us, with 1024 threads 154; 512 of
    // 16384: 63 and 68; 152 of 12288, 2048 kept: 87 and 78); of few lists the large ones (16 of 8192: 18.6 us, 24.8; of 1024: 16.5, 14.5).
    const bool few = lists <= sms;
    if (few && most <= 8192 && keep <= 512) {
        TIGA_CUDA_TRY((launch_select<SELECT_FEW, 1, true>(p, most, lists, s)));
        return launch_status();
    }
    if (lists * SELECT_CLUSTER <= 2 * sms && most > SELECT_HELD) TIGA_CUDA_TRY((launch_select<SELECT_FEW, SELECT_CLUSTER, false>(p, most, lists, s)));
    else if (few || most > 12288) TIGA_CUDA_TRY((launch_select<SELECT_FEW, 1, false>(p, most, lists, s)));
    else TIGA_CUDA_TRY((launch_select<SELECT_MANY, 1, false>(p, most, lists, s)));
    const long long tasks = lists * ((keep + 31) / 32);
    const long long grid = (tasks + MOVE_THREADS / 32 - 1) / (MOVE_THREADS / 32);
    if (grid > 0x7fffffffLL) return TIGA_ERR_UNSUPPORTED;
    TIGA_CUDA_TRY(launch_after(evict_move_kernel, dim3((unsigned)grid), MOVE_THREADS, 0, s, p, tasks));
    return launch_status();
}
