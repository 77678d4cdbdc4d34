// C-ABI entry points of the operators on rows of logits: argument checks and
// asynchronous launches (one, but for long or very many rows); nothing is allocated
// and nothing waited for.
#include "rows.h"

#include <cmath>

using namespace hbsjd;

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 40;

bool elem_ok(int32_t e) { return e == HBSJD_ELEM_F32 || e == HBSJD_ELEM_BF16 || e == HBSJD_ELEM_F16; }
bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// null, or why a [rows][V] matrix cannot be taken
const char* matrix_problem(const void* p, int32_t elem, int64_t ld, int32_t V) {
    if (!elem_ok(elem)) return "unknown element type";
    if (!p) return "NULL buffer";
    if (!aligned(p, elem_size(elem))) return "buffer not aligned to its elements";
    if (ld < V || ld > kMaxStride) return "row stride below V or above 2^40";
    return nullptr;
}

const char* rows_problem(int64_t rows, int32_t V) {
    if (rows < 0 || rows > INT32_MAX) return "need 0 <= rows < 2^31";
    if (V < 1 || V > HBSJD_ROWS_MAX_VOCAB) return "need V in [1, 262144]";
    return nullptr;
}

const char* workspace_problem(const void* p, uint64_t bytes, uint64_t need) {
    if (need && (!p || bytes < need)) return "workspace smaller than the call needs";
    if (need && !aligned(p, 16)) return "workspace not aligned to 16 bytes";
    return nullptr;
}

bool temperature_ok(float t) { return t >= 1e-6f && t <= 1e6f; }

hbsjd_status launched(const char* where) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return api_fail(HBSJD_EHIP, std::string(where) + ": " + hipGetErrorString(e));
    return HBSJD_OK;
}

}  // namespace

extern "C" {

uint64_t hbsjd_top_logits_workspace(int64_t rows, int32_t V, int32_t elem, int32_t K) {
    if (rows < 1 || rows_problem(rows, V) || !elem_ok(elem) || K < 1 || K > V || K > HBSJD_TOP_MAX)
        return 0;
    return top_logits_workspace(rows, V, K, elem);
}

uint64_t hbsjd_distill_top_workspace(int64_t rows, int32_t V, int32_t elem, int32_t K) {
    if (rows < 1 || rows_problem(rows, V) || !elem_ok(elem) || K < 1 || K > HBSJD_TOP_MAX) return 0;
    return distill_top_workspace(rows, V, K, elem);
}

hbsjd_status hbsjd_top_logits_rows(int64_t rows, int32_t V, const void* logits, int32_t elem,
                                   int64_t ld, int32_t K, float temperature, float* values,
                                   int32_t* index, float* rest, void* workspace,
                                   uint64_t workspace_bytes, void* stream) {
    try {
        if (const char* why = rows_problem(rows, V)) return api_fail(HBSJD_EINVAL, why);
        if (K < 1 || K > V || K > HBSJD_TOP_MAX)
            return api_fail(HBSJD_EINVAL, "need K in [1, min(V, 2048)]");
        if (!temperature_ok(temperature))
            return api_fail(HBSJD_EINVAL, "need a temperature in [1e-6, 1e6]");
        if (!elem_ok(elem)) return api_fail(HBSJD_EINVAL, "unknown element type");
        if (rows == 0) return HBSJD_OK;
        if (const char* why = matrix_problem(logits, elem, ld, V)) return api_fail(HBSJD_EINVAL, why);
        if (!values || !index || !rest) return api_fail(HBSJD_EINVAL, "NULL buffer");
        if (!aligned(values, 4) || !aligned(index, 4) || !aligned(rest, 4))
            return api_fail(HBSJD_EINVAL, "buffer not aligned to its elements");
        if (const char* why = workspace_problem(workspace, workspace_bytes,
                                                top_logits_workspace(rows, V, K, elem)))
            return api_fail(HBSJD_EINVAL, why);
        TopArgs a{rows, V, K, logits, elem, ld, 1.0 / temperature, values, index, rest};
        top_logits(a, workspace, (hipStream_t)stream);
        return launched("top_logits_rows");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_top_logits_rows");
    }
}

hbsjd_status hbsjd_distill_top_rows(const hbsjd_distill_args* p, float* loss, void* grad,
                                    int64_t ld_grad, void* workspace, uint64_t workspace_bytes,
                                    void* stream) {
    try {
        if (!p) return api_fail(HBSJD_EINVAL, "args is NULL");
        if (const char* why = rows_problem(p->rows, p->V)) return api_fail(HBSJD_EINVAL, why);
        if (p->K < 1 || p->K > HBSJD_TOP_MAX) return api_fail(HBSJD_EINVAL, "need K in [1, 2048]");
        if (!temperature_ok(p->temperature))
            return api_fail(HBSJD_EINVAL, "need a temperature in [1e-6, 1e6]");
        const float alpha = p->forward_weight, beta = p->reverse_weight;
        if (!(alpha >= 0.f && alpha <= 1e6f && beta >= 0.f && beta <= 1e6f && alpha + beta > 0.f))
            return api_fail(HBSJD_EINVAL, "need weights in [0, 1e6], not both 0");
        if (!elem_ok(p->elem)) return api_fail(HBSJD_EINVAL, "unknown element type");
        if (p->rows == 0) return HBSJD_OK;
        if (const char* why = matrix_problem(p->logits, p->elem, p->ld, p->V))
            return api_fail(HBSJD_EINVAL, why);
        if (!p->values || !p->index) return api_fail(HBSJD_EINVAL, "NULL buffer");
        if (beta > 0.f && !p->rest)
            return api_fail(HBSJD_EINVAL, "the reverse divergence needs rest: without it the teacher "
                                          "gives the unlisted entries no mass");
        if (!loss && !grad) return api_fail(HBSJD_EINVAL, "neither loss nor grad");
        if (!aligned(p->values, 4) || !aligned(p->index, 4) || !aligned(p->rest, 4) ||
            !aligned(p->row_weight, 4) || !aligned(loss, 4))
            return api_fail(HBSJD_EINVAL, "buffer not aligned to its elements");
        if (grad) {
            if (const char* why = matrix_problem(grad, p->elem, ld_grad, p->V))
                return api_fail(HBSJD_EINVAL, std::string("grad: ") + why);
            if (grad == p->logits && ld_grad != p->ld)
                return api_fail(HBSJD_EINVAL, "grad may be the logits only with their row stride");
        }
        if (const char* why = workspace_problem(
                workspace, workspace_bytes, distill_top_workspace(p->rows, p->V, p->K, p->elem)))
            return api_fail(HBSJD_EINVAL, why);
        const double log2_tau = 1.4426950408889634074 / (double)p->temperature;
        float log2_hi = (float)log2_tau;   // rounded down: the rest is positive
        if ((double)log2_hi >= log2_tau) log2_hi = std::nextafterf(log2_hi, 0.f);
        const float log2_lo = (float)(log2_tau - (double)log2_hi);
        DistillArgs a{p->rows, p->V, p->K, p->logits, p->elem, p->ld, p->values, p->index, p->rest,
                      1.f / p->temperature, 1.0 / p->temperature, make_float2(log2_hi, log2_lo),
                      alpha, beta, p->row_weight, loss, grad, ld_grad};
        distill_top(a, workspace, (hipStream_t)stream);
        return launched("distill_top_rows");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_distill_top_rows");
    }
}

hbsjd_status hbsjd_adjust_rows(const hbsjd_adjust_args* p, void* out, int32_t out_elem,
                               int64_t ld_out, void* stream) {
    try {
        if (!p) return api_fail(HBSJD_EINVAL, "args is NULL");
        if (const char* why = rows_problem(p->rows, p->V)) return api_fail(HBSJD_EINVAL, why);
        if (!elem_ok(p->elem)) return api_fail(HBSJD_EINVAL, "unknown element type");
        if (out_elem != p->elem && out_elem != HBSJD_ELEM_F32)
            return api_fail(HBSJD_EINVAL, "out must be fp32 or of the logits' type");
        if (p->n_tokens < 0 || p->n_bias < 0 || p->n_masks < 0)
            return api_fail(HBSJD_EINVAL, "negative list length");
        if (p->n_bias > HBSJD_ADJUST_MAX_BIASES) return api_fail(HBSJD_EINVAL, "more than 1024 biases");
        if (p->rows == 0) return HBSJD_OK;
        if (const char* why = matrix_problem(p->logits, p->elem, p->ld, p->V))
            return api_fail(HBSJD_EINVAL, why);
        if (const char* why = matrix_problem(out, out_elem, ld_out, p->V))
            return api_fail(HBSJD_EINVAL, std::string("out: ") + why);
        if (out == p->logits && (ld_out != p->ld || out_elem != p->elem))
            return api_fail(HBSJD_EINVAL, "out may be the logits only with their type and row stride");
        const bool penalties = p->repetition || p->presence || p->frequency;
        if (penalties && !p->tokens && p->n_tokens > 0)
            return api_fail(HBSJD_EINVAL, "penalties without tokens");
        if (p->n_bias > 0 && (!p->bias_index || !p->bias_value))
            return api_fail(HBSJD_EINVAL, "biases without their buffers");
        if (p->mask && p->n_masks < 1) return api_fail(HBSJD_EINVAL, "mask without masks");
        if (p->mask && !p->mask_row && p->n_masks < p->rows)
            return api_fail(HBSJD_EINVAL, "fewer masks than rows, and no mask_row");
        if (p->mask_row && !p->mask) return api_fail(HBSJD_EINVAL, "mask_row without masks");
        if (p->ld_tokens < 0 || p->ld_tokens > kMaxStride || p->ld_bias < 0 || p->ld_bias > kMaxStride)
            return api_fail(HBSJD_EINVAL, "list stride out of range");
        if (!aligned(p->tokens, 4) || !aligned(p->token_count, 4) || !aligned(p->repetition, 4) ||
            !aligned(p->presence, 4) || !aligned(p->frequency, 4) || !aligned(p->bias_index, 4) ||
            !aligned(p->bias_value, 4) || !aligned(p->mask, 4) || !aligned(p->mask_row, 4))
            return api_fail(HBSJD_EINVAL, "buffer not aligned to its elements");
        // without a penalty the histories change nothing and are not read
        AdjustArgs a{p->rows, p->V, p->logits, p->elem, p->ld, out, out_elem, ld_out,
                     penalties && p->n_tokens > 0 ? p->tokens : nullptr, p->n_tokens, p->ld_tokens,
                     p->token_count, p->repetition, p->presence, p->frequency, p->bias_index,
                     p->bias_value, p->n_bias, p->ld_bias, p->mask, p->n_masks, p->mask_row};
        adjust_rows(a, (hipStream_t)stream);
        return launched("adjust_rows");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_adjust_rows");
    }
}

}  // extern "C"
