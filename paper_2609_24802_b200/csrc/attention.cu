// Online-softmax reducer over dense and paged relations: entry points; gradients by a warp per row or per key.
#include "attention_shared.cuh"

namespace tiga {

constexpr int ATTN_WARPS = 4;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
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

template <typename T>
__device__ __forceinline__ void load4(const T* base, int D, int lane, float (&r)[4]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) r[c] = lane + 32 * c < D ? Half<T>::to(base[lane + 32 * c]) : 0.f;
}
__device__ __forceinline__ float dot4(const float (&a)[4], const float (&b)[4]) {
    return warp_sum(a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]);
}

template <typename T>
__global__ void attn_grad_q_kernel(const AttnParams p) {
    const long long w = (long long)blockIdx.x * ATTN_WARPS + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (w >= (long long)p.n_q * p.heads) return;
    const int i = (int)(w / p.heads), h = (int)(w % p.heads), hk = h / p.group;
    const int s = segment_of_row(p.q_start, p.n_seg, p.n_q, i);
    if (s < 0) return;
    const Segment g = segment_of(p, s);
    float q[4], go[4], o[4], a[4] = {0, 0, 0, 0};
    load4((const T*)p.q + i * p.q_row + h * p.q_head, p.D, lane, q);
    load4((const T*)p.go + i * p.go_row + h * p.go_head, p.D, lane, go);
    load4((const T*)p.o + w * p.D, p.D, lane, o);
    const float delta = dot4(go, o), lse = p.lse_in[w];
    for (int j = 0; j < g.nk; ++j) {
        if (p.mask && !p.mask[g.k0 + j]) continue;
        float k[4], v[4];
        load4((const T*)p.k + (g.k0 + j) * p.k_row + hk * p.k_head, p.D, lane, k);
        load4((const T*)p.v + (g.k0 + j) * p.v_row + hk * p.v_head, p.D, lane, v);
        const float ds = exp2f((dot4(q, k) * p.scale - lse) * LOG2E_F) * (dot4(go, v) - delta) * p.scale;
#pragma unroll
        for (int x = 0; x < 4; ++x) a[x] += ds * k[x];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (lane + 32 * x < p.D) ((T*)p.gq)[w * p.D + lane + 32 * x] = Half<T>::from(a[x]);
}

template <typename T>
__global__ void attn_grad_kv_kernel(const AttnParams p) {
    const long long w = (long long)blockIdx.x * ATTN_WARPS + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (w >= (long long)p.n_kv * p.kv_heads) return;
    const int j = (int)(w / p.kv_heads), hk = (int)(w % p.kv_heads);
    const int s = segment_of_row(p.kv_start, p.n_seg, p.n_kv, j);
    if (s < 0) return;
    const Segment g = segment_of(p, s);
    float k[4], v[4], a[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
    load4((const T*)p.k + j * p.k_row + hk * p.k_head, p.D, lane, k);
    load4((const T*)p.v + j * p.v_row + hk * p.v_head, p.D, lane, v);
    const bool on = !p.mask || p.mask[j];
    for (int i = g.q0; on && i < g.q0 + g.nq; ++i)
        for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
            const long long r = (long long)i * p.heads + h;
            float q[4], go[4], o[4];
            load4((const T*)p.q + i * p.q_row + h * p.q_head, p.D, lane, q);
            load4((const T*)p.go + i * p.go_row + h * p.go_head, p.D, lane, go);
            load4((const T*)p.o + r * p.D, p.D, lane, o);
            const float pr = exp2f((dot4(q, k) * p.scale - p.lse_in[r]) * LOG2E_F);
            const float ds = pr * (dot4(go, v) - dot4(go, o)) * p.scale;
#pragma unroll
            for (int x = 0; x < 4; ++x) { a[x] += ds * q[x]; b[x] += pr * go[x]; }
        }
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (lane + 32 * x < p.D) {
            if (p.gk) ((T*)p.gk)[w * p.D + lane + 32 * x] = Half<T>::from(a[x]);
            if (p.gv) ((T*)p.gv)[w * p.D + lane + 32 * x] = Half<T>::from(b[x]);
        }
}

static unsigned warps_grid(long long n) { return (unsigned)((n + ATTN_WARPS - 1) / ATTN_WARPS); }

template <typename T>
static tiga_status attn_backward(const AttnParams& p, void*, cudaStream_t s) {
    if (p.gq && p.n_q) attn_grad_q_kernel<T><<<counted(warps_grid((long long)p.n_q * p.heads)), ATTN_WARPS * 32, 0, s>>>(p);
    if ((p.gk || p.gv) && p.n_kv) attn_grad_kv_kernel<T><<<counted(warps_grid((long long)p.n_kv * p.kv_heads)), ATTN_WARPS * 32, 0, s>>>(p);
    return launch_status();
}

// ------------------------------------------------------------------------------------------------ host checks

bool attention_bad_stride(const tiga_stride& s) { return s.row < 0 || s.head < 0 || (s.row & 7) || (s.head & 7); }

tiga_status attention_heads_check(const tiga_heads* h) {
    if (!h || h->heads < 1 || h->kv_heads < 1 || h->heads % h->kv_heads || h->D < 1 || !isfinite(h->scale)) return TIGA_ERR_INVALID_ARG;
    if (h->dtype != TIGA_F32 && h->dtype != TIGA_F16 && h->dtype != TIGA_BF16) return TIGA_ERR_INVALID_ARG;
    if (h->dtype == TIGA_F32 || (h->D & 7) || h->D > 128 || h->heads > 65535) return TIGA_ERR_UNSUPPORTED;
    return TIGA_OK;
}

static AttnParams heads_params(const tiga_heads* h) {
    AttnParams p{};
    p.heads = h->heads; p.kv_heads = h->kv_heads; p.group = h->heads / h->kv_heads; p.D = h->D; p.scale = h->scale;
    p.q_row = h->q.row; p.q_head = h->q.head; p.k_row = h->key.row; p.k_head = h->key.head;
    p.v_row = h->value.row; p.v_head = h->value.head; p.go_row = h->grad_out.row; p.go_head = h->grad_out.head;
    return p;
}

// row numbers of a head group's packed rows (row * group + member) are 32-bit, and so are the counts of tiles
static bool too_many_rows(int64_t n, const tiga_heads* h) { return n * (h->heads / h->kv_heads) > 0x7fff0000LL; }

static tiga_status dense_check(const tiga_dense* g, const tiga_heads* h, AttnParams* p) {
    tiga_status st = attention_heads_check(h);
    if (st != TIGA_OK) return st;
    if (!g || g->n_seg < 0 || g->n_q < 0 || g->n_kv < 0) return TIGA_ERR_INVALID_ARG;
    if (g->n_seg > (1 << 24) || g->n_q > 0x7fffffffLL || g->n_kv > 0x7fffffffLL || too_many_rows(g->n_q, h)) return TIGA_ERR_UNSUPPORTED;
    *p = heads_params(h);
    p->q_start = g->q_start; p->kv_start = g->kv_start; p->mask = g->kv_mask;
    p->n_seg = (int)g->n_seg; p->n_q = (int)g->n_q; p->n_kv = (int)g->n_kv;
    return TIGA_OK;
}

tiga_status attention_pages_check(const tiga_pages* c) {
    if (!c || c->n_seg < 0 || c->n_pages < 0 || c->page_size < 1 || c->max_pages < 0 || c->table_stride < 0) return TIGA_ERR_INVALID_ARG;
    if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0 || ((c->page_stride | c->slot_stride | c->head_stride) & 7)) return TIGA_ERR_INVALID_ARG;
    if (c->n_seg > (1 << 24) || c->n_pages > 0x7fffffffLL || c->page_size > (1 << 24) || c->max_pages > 0x7fffffffLL) return TIGA_ERR_UNSUPPORTED;
    return TIGA_OK;
}

static tiga_status paged_check(const tiga_pages* c, const tiga_heads* h, int64_t n_q, AttnParams* p) {
    tiga_status st = attention_heads_check(h);
    if (st != TIGA_OK) return st;
    if ((st = attention_pages_check(c)) != TIGA_OK) return st;
    if (n_q < 0) return TIGA_ERR_INVALID_ARG;
    if (n_q > 0x7fffffffLL || too_many_rows(n_q, h)) return TIGA_ERR_UNSUPPORTED;
    *p = heads_params(h);
    p->k = c->key; p->v = c->value; p->table = c->table; p->kv_len = c->kv_len;
    p->k_head = p->v_head = c->head_stride;
    p->n_seg = (int)c->n_seg; p->n_q = (int)n_q;
    p->n_pages = c->n_pages; p->page_size = c->page_size; p->table_stride = c->table_stride; p->max_pages = c->max_pages;
    p->page_stride = c->page_stride; p->slot_stride = c->slot_stride;
    return TIGA_OK;
}

static bool bad_array(const void* p) { return !p || !aligned16(p); }
static bool bad_ints(const void* p) { return !p || (reinterpret_cast<uintptr_t>(p) & 3); }

}  // namespace tiga

using namespace tiga;

extern "C" size_t tiga_dense_attention_workspace_bytes(const tiga_dense* g, const tiga_heads* h, int backward) {
    AttnParams p;
    if (dense_check(g, h, &p) != TIGA_OK) return 0;
    return (backward ? 0 : attention_forward_bytes(p)) + 256;
}

extern "C" tiga_status tiga_apply_dense_attention(const tiga_dense* g, const tiga_heads* h, const void* q, const void* key, const void* value,
                                                  void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    AttnParams p;
    tiga_status st = dense_check(g, h, &p);
    if (st != TIGA_OK) return st;
    if (attention_bad_stride(h->q) || attention_bad_stride(h->key) || attention_bad_stride(h->value)) return TIGA_ERR_INVALID_ARG;
    if (g->n_seg == 0 || g->n_q == 0) return TIGA_OK;
    if (bad_ints(g->q_start) || bad_ints(g->kv_start) || bad_array(q) || bad_array(out)) return TIGA_ERR_INVALID_ARG;
    if (g->n_kv > 0 && (bad_array(key) || bad_array(value))) return TIGA_ERR_INVALID_ARG;
    if (lse && !aligned16(lse)) return TIGA_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < tiga_dense_attention_workspace_bytes(g, h, 0)) return TIGA_ERR_WORKSPACE;
    p.q = q; p.k = key; p.v = value; p.out = out; p.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return attention_forward(p, h->dtype == TIGA_BF16, ws, s);
}

extern "C" tiga_status tiga_apply_dense_attention_backward(const tiga_dense* g, const tiga_heads* h, const void* q, const void* key,
                                                           const void* value, const void* out, const float* lse, const void* grad_out,
                                                           void* grad_q, void* grad_key, void* grad_value,
                                                           void* ws, size_t ws_bytes, void* stream) {
    AttnParams p;
    tiga_status st = dense_check(g, h, &p);
    if (st != TIGA_OK) return st;
    if (attention_bad_stride(h->q) || attention_bad_stride(h->key) || attention_bad_stride(h->value) || attention_bad_stride(h->grad_out)) return TIGA_ERR_INVALID_ARG;
    if (g->n_seg == 0 || (g->n_q == 0 && g->n_kv == 0)) return TIGA_OK;
    if (!grad_q && !grad_key && !grad_value) return TIGA_OK;
    if (bad_ints(g->q_start) || bad_ints(g->kv_start)) return TIGA_ERR_INVALID_ARG;
    if (g->n_q > 0 && (bad_array(q) || bad_array(out) || bad_array(lse) || bad_array(grad_out))) return TIGA_ERR_INVALID_ARG;
    if (g->n_kv > 0 && (bad_array(key) || bad_array(value))) return TIGA_ERR_INVALID_ARG;
    if (!aligned16(grad_q) || !aligned16(grad_key) || !aligned16(grad_value)) return TIGA_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < tiga_dense_attention_workspace_bytes(g, h, 1)) return TIGA_ERR_WORKSPACE;
    p.q = q; p.k = key; p.v = value; p.o = out; p.lse_in = lse; p.go = grad_out;
    p.gq = grad_q; p.gk = grad_key; p.gv = grad_value;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return h->dtype == TIGA_F16 ? attn_backward<__half>(p, ws, s) : attn_backward<__nv_bfloat16>(p, ws, s);
}

extern "C" size_t tiga_paged_attention_workspace_bytes(const tiga_pages* c, const tiga_heads* h, int64_t n_q) {
    AttnParams p;
    if (paged_check(c, h, n_q, &p) != TIGA_OK) return 0;
    return attention_forward_bytes(p) + 256;
}

extern "C" tiga_status tiga_apply_paged_attention(const tiga_pages* c, const tiga_heads* h, const void* q, const int32_t* q_start, int64_t n_q,
                                                  int causal, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    AttnParams p;
    tiga_status st = paged_check(c, h, n_q, &p);
    if (st != TIGA_OK) return st;
    if (attention_bad_stride(h->q)) return TIGA_ERR_INVALID_ARG;
    if (c->n_seg == 0 || n_q == 0) return TIGA_OK;
    if (bad_ints(q_start) || bad_ints(c->kv_len) || bad_array(q) || bad_array(out)) return TIGA_ERR_INVALID_ARG;
    if (bad_ints(c->table) || (c->n_pages > 0 && (bad_array(c->key) || bad_array(c->value)))) return TIGA_ERR_INVALID_ARG;
    if (lse && !aligned16(lse)) return TIGA_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < tiga_paged_attention_workspace_bytes(c, h, n_q)) return TIGA_ERR_WORKSPACE;
    p.q = q; p.q_start = q_start; p.causal = causal != 0; p.out = out; p.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return attention_forward(p, h->dtype == TIGA_BF16, ws, s);
}
