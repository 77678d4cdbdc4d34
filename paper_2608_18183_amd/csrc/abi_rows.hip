// C-ABI entry points of the operators on rows of logits: argument checks and
// asynchronous launches (one, but for long or very many rows); nothing is allocated
// and nothing waited for.
#include "abi_checks.h"

using namespace hbsjd;

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
        DistillArgs a{p->rows, p->V, p->K, p->logits, p->elem, p->ld, p->values, p->index, p->rest,
                      1.f / p->temperature, 1.0 / p->temperature, log2_over(p->temperature),
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
