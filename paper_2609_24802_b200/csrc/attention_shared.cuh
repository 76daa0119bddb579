// Attention over dense and paged relations: what the kernels and the host share.
#pragma once
#include <cuda_bf16.h>
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
    int n_seg, n_q, n_kv, heads, kv_heads, group, D, causal;
    long long n_pages, page_size, table_stride, max_pages, page_stride, slot_stride;
    float scale;
};

// A segment's rows [q0, q0 + nq) and its keys [k0, k0 + nk) (paged: k0 = 0), bounds clamped to the arrays.
struct Segment { int q0, nq, k0, nk; };

__device__ __forceinline__ int clamp_to(int v, int hi) { return min(max(v, 0), hi); }

__device__ __forceinline__ Segment segment_of(const AttnParams& p, int s) {
    Segment g;
    g.q0 = clamp_to(p.q_start[s], p.n_q);
    g.nq = max(clamp_to(p.q_start[s + 1], p.n_q) - g.q0, 0);
    if (p.table) {
        g.k0 = 0;
        g.nk = (int)min((long long)max(p.kv_len[s], 0), p.max_pages * p.page_size);
    } else {
        g.k0 = clamp_to(p.kv_start[s], p.n_kv);
        g.nk = max(clamp_to(p.kv_start[s + 1], p.n_kv) - g.k0, 0);
    }
    return g;
}

// Where key j of segment s lies: its row offset in the key array (elements), or -1 where it is masked or has no page.
// (Both arrays of a paged cache share their strides; the dense value row is row(j) * v_row.)
__device__ __forceinline__ long long paged_offset(const AttnParams& p, int s, int j) {
    const int page = j / (int)p.page_size;
    const int id = p.table[(long long)s * p.table_stride + page];
    if (id < 0 || id >= p.n_pages) return -1;
    return (long long)id * p.page_stride + (long long)(j - page * (int)p.page_size) * p.slot_stride;
}

// keys that row t of the segment's nq rows reads: [0, this)
__device__ __forceinline__ int keys_of_row(const AttnParams& p, const Segment& g, int t) {
    return p.causal ? max(g.nk - g.nq + t + 1, 0) : g.nk;
}

// host checks of the descriptors (attention.cu)
tiga_status attention_heads_check(const tiga_heads* h);
tiga_status attention_pages_check(const tiga_pages* c);
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
