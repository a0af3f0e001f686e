// extern "C" entry points of the serving operators: argument checks, workspace, dispatch.
#include <cmath>

#include "kv4_attend.cuh"

namespace hbfp {

int64_t int8_pitch(int64_t k);
int launch_int8_quantize(const void* x, int dtype, int64_t d0, int64_t d1, int64_t ld, int axis, int8_t* q, int64_t pitch, float* scale, cudaStream_t st);
int launch_int8_gemm(int64_t M, int64_t N, int64_t K, const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb, const float* sb,
                     const float* bias, void* y, int dtype, int64_t ldy, cudaStream_t st);
// One to three tokens, converted by the product's launch (int8_few.cu).
bool int8_few_eligible(int64_t M, int64_t K);
int launch_int8_few(int64_t M, int64_t N, int64_t K, const void* a, int a_dtype, int64_t lda, const float* sa, const int8_t* w, int64_t ldw, const float* sw,
                    const float* bias, void* y, int dtype, int64_t ldy, cudaStream_t st);
int launch_kv4_append(const Kv4Args& a, int dtype, const void* k, Kv4Rows ks, const void* v, Kv4Rows vs, cudaStream_t st);
int launch_kv4_read(const Kv4Args& a, int count, float* k, float* v, cudaStream_t st);

namespace {

constexpr int64_t INT8_MOST_K = 131072;              // 128 * 128 * K fits int32
constexpr float LOG2_E = 1.4426950408889634f;
constexpr int64_t MOST = 1ll << 30;                  // extents the kernels index with 32 bits

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether two matrices of `rows` rows surely share bytes: their ranges meet and, with more than one row, their rows, equally far apart, do.
bool share_bytes(const void* a, int64_t a_row, int64_t a_pitch, const void* b, int64_t b_row, int64_t b_pitch, int64_t rows) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    if (pa + ((rows - 1) * a_pitch + a_row) <= pb || pb + ((rows - 1) * b_pitch + b_row) <= pa) return false;
    if (rows == 1) return true;
    if (a_pitch != b_pitch) return false;
    const int64_t d = pb >= pa ? (int64_t)((pb - pa) % a_pitch) : (a_pitch - (int64_t)((pa - pb) % a_pitch)) % a_pitch;      // columns from a's to b's
    return d < a_row || d + b_row > a_pitch;
}

int kv4_args(const hbfp_kv4_cache* c, const hbfp_kv4_batch* b, Kv4Args* a) {
    if (!c || !b || c->struct_size != sizeof(*c) || b->struct_size != sizeof(*b)) return HBFP_ERR_INVALID_ARG;
    if (c->heads < 1 || c->pages < 0 || b->sequences < 0 || b->tokens < 0 || b->max_tokens < 0 || b->table_pages < 0 || b->table_ld < b->table_pages)
        return HBFP_ERR_INVALID_ARG;
    if (c->page < 16 || (c->page & (c->page - 1)) != 0) return HBFP_ERR_UNSUPPORTED;
    if (c->dim != 64 && c->dim != 96 && c->dim != 128 && c->dim != 256) return HBFP_ERR_UNSUPPORTED;
    // grid extents, and positions, which are 32-bit numbers
    if (c->heads > 65535 || b->sequences > 65535 || b->tokens >= MOST || (int64_t)b->table_pages * c->page >= MOST) return HBFP_ERR_UNSUPPORTED;
    if (c->pages > 0 && (!c->k_mant || !c->k_exps || !c->v_mant || !c->v_exps)) return HBFP_ERR_INVALID_ARG;
    if (!aligned(c->k_mant, 16) || !aligned(c->v_mant, 16) || !aligned(c->k_exps, 16) || !aligned(c->v_exps, 16)) return HBFP_ERR_ALIGNMENT;
    if (b->sequences > 0 && (!b->lengths || (b->table_pages > 0 && !b->table))) return HBFP_ERR_INVALID_ARG;
    if (!b->starts && (int64_t)b->sequences * b->max_tokens != b->tokens) return HBFP_ERR_INVALID_ARG;
    a->k_mant = c->k_mant;
    a->v_mant = c->v_mant;
    a->k_exps = c->k_exps;
    a->v_exps = c->v_exps;
    a->pages = c->pages;
    a->heads = c->heads;
    a->dim = c->dim;
    a->page = c->page;
    a->shift = 0;
    while ((1 << a->shift) < c->page) ++a->shift;
    a->table = b->table;
    a->table_ld = b->table_ld;
    a->table_pages = b->table_pages;
    a->sequences = b->sequences;
    a->lengths = b->lengths;
    a->starts = b->starts;
    a->tokens = b->tokens;
    a->most = b->max_tokens;
    a->status = nullptr;
    return HBFP_OK;
}

int attend(const hbfp_kv4_cache* cache, const hbfp_kv4_batch* batch, int dtype, int group, int window, Kv4Attend* a, cudaStream_t st, size_t* bytes) {
    if (!dtype_ok(dtype) || group < 1 || window < 0) return HBFP_ERR_INVALID_ARG;
    if (const int rc = kv4_args(cache, batch, &a->c)) return rc;
    if ((int64_t)a->c.heads * group > 65535 || (int64_t)a->c.most * group >= MOST) return HBFP_ERR_UNSUPPORTED;
    a->group = group;
    a->window = (int)(window < MOST ? window : MOST);
    if (bytes) *bytes = 0;
    if (a->c.sequences == 0 || a->c.most == 0 || a->c.tokens == 0) return HBFP_OK;
    if (!bytes) {
        a->c.status = device_status_word();
        if (!a->c.status) return HBFP_ERR_CUDA;
    }
    if (kv4_prompt_eligible(*a, dtype)) return bytes ? (int)HBFP_OK : launch_kv4_prompt(*a, dtype, st);
    if (dtype == HBFP_F32) return launch_kv4_attend_f32(*a, st, bytes);
    if (dtype == HBFP_BF16) return launch_kv4_attend_bf16(*a, st, bytes);
    return launch_kv4_attend_f16(*a, st, bytes);
}

}  // namespace
}  // namespace hbfp

using namespace hbfp;

extern "C" {

int hbfp_int8_quantize(const void* x, int dtype, int64_t d0, int64_t d1, int64_t ld, int contract_axis, int8_t* q, int64_t pitch, float* scale, void* stream) {
    if (!dtype_ok(dtype) || d0 < 0 || d1 < 0 || ld < d1 || (contract_axis != 0 && contract_axis != 1)) return HBFP_ERR_INVALID_ARG;
    const int64_t rows = contract_axis == 1 ? d0 : d1, k = contract_axis == 1 ? d1 : d0;
    if (pitch < k || pitch < 16) return HBFP_ERR_INVALID_ARG;
    if (rows >= MOST || k >= MOST || pitch >= 2 * MOST) return HBFP_ERR_UNSUPPORTED;
    if (rows > 0 && (!q || !scale || (k > 0 && !x))) return HBFP_ERR_INVALID_ARG;
    if (pitch % 16 != 0 || !aligned(q, 16)) return HBFP_ERR_ALIGNMENT;
    return launch_int8_quantize(x, dtype, d0, d1, ld, contract_axis, q, pitch, scale, static_cast<cudaStream_t>(stream));
}

int hbfp_int8_gemm_workspace(int64_t M, int64_t N, int64_t K, int a_dtype, size_t* bytes) {
    if (!bytes || M < 0 || N < 0 || K < 0 || (a_dtype != HBFP_I8 && !dtype_ok(a_dtype))) return HBFP_ERR_INVALID_ARG;
    if (K >= INT8_MOST_K || M >= MOST || N >= MOST) return HBFP_ERR_UNSUPPORTED;
    *bytes = a_dtype == HBFP_I8 || M == 0 || N == 0 || K == 0 || int8_few_eligible(M, K) ? 0 : (size_t)(round_up(M * int8_pitch(K), 256) + 4 * M);
    return HBFP_OK;
}

int hbfp_int8_gemm(int64_t M, int64_t N, int64_t K, const void* a, int a_dtype, int64_t lda, const float* a_scale, const int8_t* w, int64_t ldw,
                   const float* w_scale, const float* bias, void* y, int y_dtype, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    const int rc = hbfp_int8_gemm_workspace(M, N, K, a_dtype, &need);
    if (rc) return rc;
    if (!dtype_ok(y_dtype) || ldy < N || lda < K || ldw < K) return HBFP_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return HBFP_OK;
    if (!y || !w_scale || (K > 0 && (!a || !w))) return HBFP_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int8_t* qa = static_cast<const int8_t*>(a);
    if (K > 0) {
        if (ldw % 16 != 0 || !aligned(w, 16)) return HBFP_ERR_ALIGNMENT;
        if (a_dtype == HBFP_I8) {
            if (!a_scale) return HBFP_ERR_INVALID_ARG;
            if (lda % 16 != 0 || !aligned(a, 16)) return HBFP_ERR_ALIGNMENT;
        }
        const int64_t a_bytes = a_dtype == HBFP_I8 ? 1 : dtype_bytes(a_dtype), y_bytes = dtype_bytes(y_dtype);
        // (activations that are converted first have been read when the product stores)
        if (need == 0 && share_bytes(a, K * a_bytes, lda * a_bytes, y, N * y_bytes, ldy * y_bytes, M)) return HBFP_ERR_INVALID_ARG;
        if (int8_few_eligible(M, K)) return launch_int8_few(M, N, K, a, a_dtype, lda, a_scale, w, ldw, w_scale, bias, y, y_dtype, ldy, st);
        if (a_dtype != HBFP_I8) {
            if (!workspace || workspace_bytes < need) return HBFP_ERR_WORKSPACE;
            if (!aligned(workspace, 256)) return HBFP_ERR_ALIGNMENT;
            const int64_t pitch = int8_pitch(K);
            int8_t* const q = static_cast<int8_t*>(workspace);
            float* const s = reinterpret_cast<float*>(q + round_up(M * pitch, 256));
            if (const int bad = launch_int8_quantize(a, a_dtype, M, K, lda, 1, q, pitch, s, st)) return bad;
            qa = q;
            lda = pitch;
            a_scale = s;
        }
    }
    return launch_int8_gemm(M, N, K, qa, lda, a_scale, w, ldw, w_scale, bias, y, y_dtype, ldy, st);
}

int hbfp_kv4_append(const hbfp_kv4_cache* cache, const hbfp_kv4_batch* batch, int dtype, const void* k, int64_t k_token, int64_t k_head, const void* v,
                    int64_t v_token, int64_t v_head, void* stream) {
    Kv4Args a;
    if (!dtype_ok(dtype)) return HBFP_ERR_INVALID_ARG;
    if (const int rc = kv4_args(cache, batch, &a)) return rc;
    if (a.sequences == 0 || a.tokens == 0 || a.most == 0) return HBFP_OK;
    if (!k || !v) return HBFP_ERR_INVALID_ARG;
    a.status = device_status_word();
    if (!a.status) return HBFP_ERR_CUDA;
    return launch_kv4_append(a, dtype, k, Kv4Rows{k_token, k_head}, v, Kv4Rows{v_token, v_head}, static_cast<cudaStream_t>(stream));
}

int hbfp_kv4_read(const hbfp_kv4_cache* cache, const hbfp_kv4_batch* batch, int32_t count, float* k, float* v, void* stream) {
    if (!batch || batch->struct_size != sizeof(*batch) || count < 0) return HBFP_ERR_INVALID_ARG;
    hbfp_kv4_batch all = *batch;
    all.starts = nullptr;
    all.max_tokens = count;
    all.tokens = (int64_t)all.sequences * count;
    Kv4Args a;
    if (const int rc = kv4_args(cache, &all, &a)) return rc;
    if (a.tokens == 0) return HBFP_OK;
    if (!k || !v) return HBFP_ERR_INVALID_ARG;
    if (!aligned(k, 32) || !aligned(v, 32)) return HBFP_ERR_ALIGNMENT;
    a.status = device_status_word();
    if (!a.status) return HBFP_ERR_CUDA;
    return launch_kv4_read(a, count, k, v, static_cast<cudaStream_t>(stream));
}

int hbfp_kv4_attention_workspace(const hbfp_kv4_cache* cache, const hbfp_kv4_batch* batch, int dtype, int32_t group, int32_t window, size_t* bytes) {
    if (!bytes) return HBFP_ERR_INVALID_ARG;
    Kv4Attend a{};
    return attend(cache, batch, dtype, group, window, &a, nullptr, bytes);
}

int hbfp_kv4_attention(const hbfp_kv4_cache* cache, const hbfp_kv4_batch* batch, int dtype, const void* q, int64_t q_token, int64_t q_head, int32_t group,
                       float scale, int32_t window, void* out, int64_t out_token, int64_t out_head, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    Kv4Attend a{};
    if (!std::isfinite(scale * LOG2_E)) return HBFP_ERR_INVALID_ARG;       // (the kernels would not agree on what it gives)
    if (const int rc = attend(cache, batch, dtype, group, window, &a, nullptr, &need)) return rc;
    if (a.c.sequences == 0 || a.c.most == 0 || a.c.tokens == 0) return HBFP_OK;
    if (!q || !out) return HBFP_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || workspace_bytes < need)) return HBFP_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return HBFP_ERR_ALIGNMENT;
    a.q = q;
    a.qs = Kv4Rows{q_token, q_head};
    a.out = out;
    a.os = Kv4Rows{out_token, out_head};
    a.scale2 = scale * LOG2_E;
    a.partial = static_cast<float*>(workspace);
    return attend(cache, batch, dtype, group, window, &a, static_cast<cudaStream_t>(stream), nullptr);
}

}  // extern "C"
