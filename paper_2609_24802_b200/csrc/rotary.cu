// Rotary positions, on their own and on the way into the pages of a cache.
//
// A pair (a, b) of features at position n is turned by t = n f: (a cos t - b sin t, a sin t + b cos t).  The work is bound by
// memory: every element is read and written once, the turn costs six operations per pair, its sine and cosine are formed once per
// (row, pair) of a block and lie in shared memory for the row's heads.
// t is a number of turns in 64-bit fixed point: f / 2 pi without its whole turns, times the position, modulo 2^64.  Whole turns drop
// out by themselves, and position 2^22 keeps an error of 2^22 2^-54 turns; the upper 32 bits, at most half a turn either way, enter
// sincospif in fp32.  (In fp32 the product alone is off by 2^22 2^-24 / 2 turns: the angle would mean nothing.  Formed once per row and
// pair of a block: formed again for every few heads they took as long as the memory.)
#include "attention_shared.cuh"

namespace tiga {

// 16384 rows of 32 heads of 128 in bf16, part of a wider array: 4.5 TB/s.
constexpr int ROT_THREADS = 256;
constexpr int ROT_ROWS = 8, ROT_PAIRS_MAX = 4096;

struct RotParams {
    const void *x, *value;          // value: append only
    void *y, *vy;
    const double* freq;
    const void* positions;
    const int32_t *start, *kv_len, *table;
    long long x_row, x_head, v_row, v_head, y_row, y_head, slot_stride, page_size, max_pages, table_stride, n_pages;
    long long n;
    int pos64, n_seg, heads, D, turned, pairs, rows, rot_units, tail_units, val_units, in_place;
    float magnitude;
    int inverse;
};

// f / 2 pi modulo a turn, in units of 2^-64 turns
__device__ __forceinline__ unsigned long long turns_of(double f) {
    double t = f * 0.15915494309189533577;
    t -= floor(t);
    return t < 1.0 ? (unsigned long long)(t * 18446744073709551616.0) : 0ull;
}
template <typename T, int VEC, bool ALIGNED>
struct alignas(ALIGNED ? sizeof(T) * VEC : sizeof(T)) Pack { T e[VEC]; };

// VEC elements at p; unaligned: those of them below `left`
template <typename T, int VEC, bool ALIGNED>
__device__ __forceinline__ Pack<T, VEC, ALIGNED> load_pack(const T* p, int left) {
    Pack<T, VEC, ALIGNED> r;
    if (ALIGNED) r = *reinterpret_cast<const Pack<T, VEC, ALIGNED>*>(p);
    else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) r.e[i] = i < left ? p[i] : T(0.f);
    }
    return r;
}
template <typename T, int VEC, bool ALIGNED>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, VEC, ALIGNED>& r, int left) {
    if (ALIGNED) *reinterpret_cast<Pack<T, VEC, ALIGNED>*>(p) = r;
    else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) if (i < left) p[i] = r.e[i];
    }
}

// A block has up to ROT_ROWS rows.  It looks up where they lie, forms the sines and cosines of their pairs once, and then passes over
// the rows' heads in the order of memory.  A unit is VEC pairs as two vectors of the halves, VEC / 2 pairs as one vector, or one vector
// of what is copied.  Many threads hide the
// loads, not batches of them: two and four units a thread at a time cost registers and 14 and 67 %.
template <typename T, int VEC, bool ALIGNED, bool APPEND>
__global__ void __launch_bounds__(ROT_THREADS, APPEND ? 6 : 8) rotary_kernel(const RotParams p) {
    extern __shared__ float2 turn[];            // [rows][pairs]: cosine, sine
    __shared__ long long position[ROT_ROWS], target[ROT_ROWS];      // target: the row's offset in y, -1: it goes nowhere
    const long long first_row = (long long)blockIdx.x * p.rows;
    const int rows = (int)min((long long)p.rows, p.n - first_row), n_pairs = p.turned / 2;
    if (threadIdx.x < rows) {
        const long long i = first_row + threadIdx.x;
        long long pos = 0, y0 = -1;
        if (APPEND) {
            const int s = segment_of_row(p.start, p.n_seg, (int)p.n, (int)i);
            if (s >= 0) {
                const int first = clamp_to(p.start[s], (int)p.n), end = clamp_to(p.start[s + 1], (int)p.n);
                pos = (long long)max(p.kv_len[s], 0) - (end - i);
                if (pos >= 0 && pos < p.max_pages * p.page_size && first <= i) {
                    const long long page = quotient(pos, p.page_size);
                    const int id = p.table[s * p.table_stride + page];
                    if (id >= 0 && id < p.n_pages) y0 = id * p.y_row + (pos - page * p.page_size) * p.slot_stride;
                }
            }
        } else {
            pos = p.pos64 ? ((const long long*)p.positions)[i] : ((const int*)p.positions)[i];
            y0 = i * p.y_row;
        }
        position[threadIdx.x] = pos;
        target[threadIdx.x] = y0;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < rows * n_pairs; k += ROT_THREADS) {
        const int r = k / n_pairs;
        const unsigned long long t = (unsigned long long)position[r] * turns_of(p.freq[k - r * n_pairs]);
        float c, s;
        sincospif((float)(int)(t >> 32) * 0x1p-31f, &s, &c);
        turn[k] = make_float2(c * p.magnitude, p.inverse ? -s * p.magnitude : s * p.magnitude);
    }
    __syncthreads();

    // A thread has one unit of every step-th (row, head); rows wider than a block are cut into parts of its threads.
    typedef Pack<T, VEC, ALIGNED> V;
    const int units = p.rot_units + (p.in_place ? 0 : p.tail_units) + (APPEND ? p.val_units : 0);
    const int part = min(units, ROT_THREADS), step = ROT_THREADS / part;
    const int lane = threadIdx.x % part, begin = threadIdx.x / part;
    if (begin >= step) return;
    for (int u = lane; u < units; u += part) {
        const bool turned = u < p.rot_units, value = APPEND && u >= p.rot_units + p.tail_units;
        const int at = turned ? u * VEC : value ? (u - p.rot_units - p.tail_units) * VEC : p.turned + (u - p.rot_units) * VEC;
        const int left = turned ? (p.pairs ? p.turned : n_pairs) - at : p.D - at;
        const T* src = (const T*)(value ? p.value : p.x) + at;
        T* dst = (T*)(value ? p.vy : p.y) + at;
        const long long src_row = value ? p.v_row : p.x_row, src_head = value ? p.v_head : p.x_head;
        for (int r = begin / p.heads, h = begin - r * p.heads; r < rows;) {
            if (target[r] >= 0) {
                const T* from = src + (first_row + r) * src_row + h * src_head;
                T* to = dst + target[r] + h * p.y_head;
                V a = load_pack<T, VEC, ALIGNED>(from, left);
                if (turned) {
                    const float2* cs = turn + r * n_pairs + (p.pairs ? at / 2 : at);
                    if (p.pairs) {
#pragma unroll
                        for (int k = 0; k < VEC / 2; ++k) {
                            const float e = Half<T>::to(a.e[2 * k]), f = Half<T>::to(a.e[2 * k + 1]);
                            const float2 t = cs[k];
                            a.e[2 * k] = Half<T>::from(e * t.x - f * t.y);
                            a.e[2 * k + 1] = Half<T>::from(e * t.y + f * t.x);
                        }
                    } else {
                        V b = load_pack<T, VEC, ALIGNED>(from + n_pairs, left);
#pragma unroll
                        for (int k = 0; k < VEC; ++k) {
                            if (!ALIGNED && k >= left) continue;
                            const float e = Half<T>::to(a.e[k]), f = Half<T>::to(b.e[k]);
                            const float2 t = cs[k];
                            a.e[k] = Half<T>::from(e * t.x - f * t.y);
                            b.e[k] = Half<T>::from(e * t.y + f * t.x);
                        }
                        store_pack<T, VEC, ALIGNED>(to + n_pairs, b, left);
                    }
                }
                store_pack<T, VEC, ALIGNED>(to, a, left);
            }
            h += step;
            while (h >= p.heads) { h -= p.heads; ++r; }
        }
    }
}

template <typename T, int VEC, bool ALIGNED, bool APPEND>
static tiga_status launch_rotary_t(RotParams p, cudaStream_t s) {
    const int np = p.pairs ? VEC / 2 : VEC;
    p.rot_units = (p.turned / 2 + np - 1) / np;
    p.tail_units = (p.D - p.turned + VEC - 1) / VEC;
    p.val_units = (p.D + VEC - 1) / VEC;
    if (APPEND == false && p.in_place && p.rot_units == 0) return TIGA_OK;
    // rows of a block: as many as leave four blocks an SM and their sines and cosines room (32 KB)
    long long rows = p.n / (148 * 4);
    const int room = p.turned ? ROT_PAIRS_MAX / (p.turned / 2) : ROT_ROWS;
    rows = rows < 1 ? 1 : rows > ROT_ROWS ? ROT_ROWS : rows;
    p.rows = (int)(rows > room ? room : rows);
    const long long blocks = (p.n + p.rows - 1) / p.rows;
    if (blocks > 0x7fffffffLL || (long long)p.rows * p.heads * (p.rot_units + p.tail_units + p.val_units) > 0x7fffffffLL) return TIGA_ERR_UNSUPPORTED;
    rotary_kernel<T, VEC, ALIGNED, APPEND><<<counted((unsigned)blocks), ROT_THREADS, (size_t)p.rows * (p.turned / 2) * sizeof(float2), s>>>(p);
    return launch_status();
}

// The widest vector that pairs, copied features, strides and bases allow: 16 bytes, 8, or element by element.
template <typename T, bool APPEND>
static tiga_status launch_rotary(const RotParams& p, cudaStream_t s) {
    constexpr int W = 16 / (int)sizeof(T);
    const uintptr_t bases = (uintptr_t)p.x | (uintptr_t)p.y | (uintptr_t)p.value | (uintptr_t)p.vy;
    const long long strides = p.x_row | p.x_head | p.y_row | p.y_head | p.v_row | p.v_head | p.slot_stride;
    auto fits = [&](int v) {
        return bases % (v * sizeof(T)) == 0 && strides % v == 0 && p.D % v == 0 && (p.pairs ? p.turned : p.turned / 2) % v == 0 && p.turned % v == 0;
    };
    if (fits(W)) return launch_rotary_t<T, W, true, APPEND>(p, s);
    if (fits(W / 2)) return launch_rotary_t<T, W / 2, true, APPEND>(p, s);
    return launch_rotary_t<T, 2, false, APPEND>(p, s);
}

static tiga_status rotary_check(const tiga_rotary* r, int32_t D) {
    if (!r || r->turned < 2 || (r->turned & 1) || r->turned > D || !isfinite(r->magnitude)) return TIGA_ERR_INVALID_ARG;
    if (r->layout != TIGA_ROT_HALVES && r->layout != TIGA_ROT_PAIRS) return TIGA_ERR_INVALID_ARG;
    return TIGA_OK;
}

}  // namespace tiga

using namespace tiga;

extern "C" tiga_status tiga_rotary_frequencies(int32_t turned, double base, int32_t scaling, double factor, double length, double slow,
                                               double fast, double* freq, float* magnitude) {
    if (turned < 2 || (turned & 1) || !(base > 0) || !isfinite(base) || !freq || !magnitude) return TIGA_ERR_INVALID_ARG;
    if (scaling < TIGA_ROT_PLAIN || scaling > TIGA_ROT_BANDS) return TIGA_ERR_INVALID_ARG;
    if (scaling != TIGA_ROT_PLAIN && (!(factor >= 1) || !isfinite(factor))) return TIGA_ERR_INVALID_ARG;
    if (scaling == TIGA_ROT_BANDS && (!(length > 0) || !(slow >= 0) || !(fast > slow) || !isfinite(length) || !isfinite(fast))) return TIGA_ERR_INVALID_ARG;
    if (scaling == TIGA_ROT_BASE && turned == 2) return TIGA_ERR_INVALID_ARG;      // a single pair turns by one radian whatever the base
    if (scaling == TIGA_ROT_BASE) base *= pow(factor, turned / (turned - 2.0));
    for (int i = 0; i < turned / 2; ++i) {
        double f = pow(base, -2.0 * i / turned);
        if (scaling == TIGA_ROT_LINEAR) f /= factor;
        if (scaling == TIGA_ROT_BANDS) {
            const double g = (length * f / 6.283185307179586477 - slow) / (fast - slow), keep = g < 0 ? 0 : g > 1 ? 1 : g;
            f = keep * f + (1 - keep) * f / factor;
        }
        freq[i] = f;
    }
    *magnitude = scaling == TIGA_ROT_BANDS ? (float)(0.1 * log(factor) + 1.0) : 1.f;
    return TIGA_OK;
}

extern "C" tiga_status tiga_apply_rotary(const tiga_rotary* r, const void* x, const tiga_stride* xs, void* y, const tiga_stride* ys,
                                         tiga_dtype dtype, int64_t n, int32_t heads, int32_t D, const void* positions, int32_t position_type,
                                         int inverse, void* stream) {
    if (D < 1 || heads < 1 || n < 0 || !xs || !ys || xs->row < 0 || xs->head < 0 || ys->row < 0 || ys->head < 0) return TIGA_ERR_INVALID_ARG;
    if (dtype != TIGA_F32 && dtype != TIGA_F16 && dtype != TIGA_BF16) return TIGA_ERR_INVALID_ARG;
    if (position_type != TIGA_I32 && position_type != TIGA_I64) return TIGA_ERR_INVALID_ARG;
    tiga_status st = rotary_check(r, D);
    if (st != TIGA_OK) return st;
    if (n == 0) return TIGA_OK;
    const uintptr_t e = dtype == TIGA_F32 ? 4 : 2;
    if (!x || !y || (uintptr_t)x % e || (uintptr_t)y % e || !r->freq || (uintptr_t)r->freq % 8) return TIGA_ERR_INVALID_ARG;
    if (!positions || (uintptr_t)positions % (position_type == TIGA_I64 ? 8 : 4)) return TIGA_ERR_INVALID_ARG;
    if (x == y && (xs->row != ys->row || xs->head != ys->head)) return TIGA_ERR_INVALID_ARG;
    // rows or heads of y that share storage would be written twice
    if ((n > 1 && ys->row == 0) || (heads > 1 && ys->head == 0)) return TIGA_ERR_INVALID_ARG;
    if (n > (1LL << 40) || r->turned > 2 * ROT_PAIRS_MAX) return TIGA_ERR_UNSUPPORTED;
    RotParams p{};
    p.x = x; p.y = y; p.x_row = xs->row; p.x_head = xs->head; p.y_row = ys->row; p.y_head = ys->head; p.in_place = x == y;
    p.freq = r->freq; p.turned = r->turned; p.pairs = r->layout == TIGA_ROT_PAIRS; p.magnitude = r->magnitude; p.inverse = inverse != 0;
    p.positions = positions; p.pos64 = position_type == TIGA_I64; p.n = n; p.heads = heads; p.D = D;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == TIGA_F32) return launch_rotary<float, false>(p, s);
    return dtype == TIGA_F16 ? launch_rotary<__half, false>(p, s) : launch_rotary<__nv_bfloat16, false>(p, s);
}

extern "C" tiga_status tiga_paged_append(const tiga_pages* c, const tiga_heads* h, const void* key, const void* value, const int32_t* start,
                                         int64_t n_new, const tiga_rotary* r, void* stream) {
    tiga_status st = attention_heads_check(h);
    if (st != TIGA_OK) return st;
    if ((st = attention_pages_check(c)) != TIGA_OK) return st;
    if (r && (st = rotary_check(r, h->D)) != TIGA_OK) return st;
    if (n_new < 0 || attention_bad_stride(h->key) || attention_bad_stride(h->value)) return TIGA_ERR_INVALID_ARG;
    if (n_new > 0x7fffffffLL) return TIGA_ERR_UNSUPPORTED;
    if (c->n_seg == 0 || n_new == 0 || c->n_pages == 0 || c->max_pages == 0) return TIGA_OK;
    // slots or heads of a page that share storage would be written twice
    if ((c->page_size > 1 && c->slot_stride == 0) || (h->kv_heads > 1 && c->head_stride == 0) || (c->n_pages > 1 && c->page_stride == 0)) return TIGA_ERR_INVALID_ARG;
    if (!key || !value || !c->key || !c->value || !aligned16(key) || !aligned16(value) || !aligned16(c->key) || !aligned16(c->value)) return TIGA_ERR_INVALID_ARG;
    if (!start || (uintptr_t)start % 4 || !c->table || (uintptr_t)c->table % 4 || !c->kv_len || (uintptr_t)c->kv_len % 4) return TIGA_ERR_INVALID_ARG;
    if (r && (!r->freq || (uintptr_t)r->freq % 8)) return TIGA_ERR_INVALID_ARG;
    RotParams p{};
    p.x = key; p.value = value; p.y = c->key; p.vy = c->value;
    p.x_row = h->key.row; p.x_head = h->key.head; p.v_row = h->value.row; p.v_head = h->value.head;
    p.y_row = c->page_stride; p.y_head = c->head_stride; p.slot_stride = c->slot_stride;
    p.page_size = c->page_size; p.max_pages = c->max_pages; p.table_stride = c->table_stride; p.n_pages = c->n_pages;
    p.start = start; p.kv_len = c->kv_len; p.table = c->table; p.n_seg = (int)c->n_seg;
    p.n = n_new; p.heads = h->kv_heads; p.D = h->D;
    if (r) { p.freq = r->freq; p.turned = r->turned; p.pairs = r->layout == TIGA_ROT_PAIRS; p.magnitude = r->magnitude; }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return h->dtype == TIGA_F16 ? launch_rotary<__half, true>(p, s) : launch_rotary<__nv_bfloat16, true>(p, s);
}
