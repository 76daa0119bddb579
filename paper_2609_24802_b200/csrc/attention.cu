// Online-softmax reducer over dense and paged relations: entry points and their checks.
#include "attention_tiles.cuh"

namespace tiga {

// ------------------------------------------------------------------------------------------------ tensor maps

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's encoder (NULL: there is none, rows are copied one by one)
static EncodeTiled encoder() {
    static const EncodeTiled f = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return (EncodeTiled) nullptr;
        }
        return (EncodeTiled)fn;
    }();
    return f;
}

// dims and strides (elements) from the features outwards; boxes of 64 features.  Strides of zero (shared storage) have no map.
static bool encode(CUtensorMap* m, bool bf16, const void* base, const long long (&dim)[4], const long long (&stride)[3], int box1, int box2) {
    cuuint64_t d[4], st[3];
    for (int i = 0; i < 4; ++i) {
        if (dim[i] < 1 || dim[i] > 0xffffffffLL) return false;
        d[i] = dim[i];
    }
    for (int i = 0; i < 3; ++i) {
        if (stride[i] <= 0 && dim[i + 1] > 1) return false;
        if (stride[i] >= 1LL << 38) return false;
        st[i] = (dim[i + 1] > 1 ? stride[i] : 64) * 2;          // (of a single entry: any)
    }
    const cuuint32_t box[4] = {64, (cuuint32_t)box1, (cuuint32_t)box2, 1}, one[4] = {1, 1, 1, 1};
    return encoder()(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), d, st, box, one,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

void make_tile_maps(AttnParams* p, bool bf16, TileMaps* m) {
    p->kv_box = p->q_box = 0;
    if (!encoder()) return;
    if (p->n_q > 0 && 32 % p->group == 0) {
        const long long dim[4] = {p->D, p->heads, p->n_q, 1};
        const bool q = encode(&m->q, bf16, p->q, dim, {p->q_head, p->q_row, 64}, p->group, 32 / p->group);
        p->q_box = q && (!p->go || encode(&m->go, bf16, p->go, dim, {p->go_head, p->go_row, 64}, p->group, 32 / p->group)) ? 32 : 0;
    }
    // pages: the rows of a box lie in one page and begin on a group of eight
    int box = 32;
    while (p->table && box >= 8 && p->page_size % box) box /= 2;
    if (box < 8) return;
    const long long dense[4] = {p->D, p->n_kv, p->kv_heads, 1}, paged[4] = {p->D, p->page_size, p->kv_heads, p->n_pages};
    const bool ok = p->table
        ? encode(&m->k, bf16, p->k, paged, {p->slot_stride, p->k_head, p->page_stride}, box, 1) && encode(&m->v, bf16, p->v, paged, {p->slot_stride, p->v_head, p->page_stride}, box, 1)
        : encode(&m->k, bf16, p->k, dense, {p->k_row, p->k_head, 64}, box, 1) && encode(&m->v, bf16, p->v, dense, {p->v_row, p->v_head, 64}, box, 1);
    p->kv_box = ok ? box : 0;
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
static bool too_many_rows(int64_t n, const tiga_heads* h) { return n * (h->heads / h->kv_heads) > MOST_ROWS; }

static tiga_status dense_check(const tiga_dense* g, const tiga_heads* h, AttnParams* p) {
    tiga_status st = attention_heads_check(h);
    if (st != TIGA_OK) return st;
    if (!g || g->n_seg < 0 || g->n_q < 0 || g->n_kv < 0) return TIGA_ERR_INVALID_ARG;
    if (g->n_seg > (1 << 24) || g->n_q > 0x7fffffffLL || g->n_kv > MOST_ROWS || too_many_rows(g->n_q, h)) return TIGA_ERR_UNSUPPORTED;
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
    return (backward ? attention_backward_bytes(p) : attention_forward_bytes(p)) + 256;
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
    return attention_backward(p, h->dtype == TIGA_BF16, ws, s);
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
    if ((c->max_pages > 0 && bad_ints(c->table)) || (c->n_pages > 0 && (bad_array(c->key) || bad_array(c->value)))) return TIGA_ERR_INVALID_ARG;
    if (lse && !aligned16(lse)) return TIGA_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < tiga_paged_attention_workspace_bytes(c, h, n_q)) return TIGA_ERR_WORKSPACE;
    if (c->max_pages == 0) p.table = c->kv_len;         // an empty table may have no address; any says that the relation is paged, and none of it is read
    p.q = q; p.q_start = q_start; p.causal = causal != 0; p.out = out; p.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return attention_forward(p, h->dtype == TIGA_BF16, ws, s);
}
