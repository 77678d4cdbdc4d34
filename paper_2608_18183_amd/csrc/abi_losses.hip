// C-ABI entry points of the operators of a policy or preference step (tokens'
// log-probabilities, losses with their gradients, norms of gradients): argument
// checks and asynchronous launches; nothing is allocated on the device and nothing
// waited for.
#include "abi_checks.h"

#include <vector>

#include "grad_norm.h"

using namespace hbsjd;

namespace {

constexpr float kMaxWeight = 1e6f;
bool weight_ok(float w) { return w >= 0.f && w <= kMaxWeight; }

// what the three calls on rows check alike
template <typename Args> const char* token_problem(const Args* p, const void* grad, int64_t ld_grad) {
    if (const char* why = matrix_problem(p->logits, p->elem, p->ld, p->V)) return why;
    if (!p->tokens) return "NULL buffer";
    if (!aligned(p->tokens, 4)) return "buffer not aligned to its elements";
    if (!grad) return nullptr;
    if (const char* why = matrix_problem(grad, p->elem, ld_grad, p->V)) return why;
    if (grad == p->logits && ld_grad != p->ld) return "grad may be the logits only with their row stride";
    return nullptr;
}

// sizes, types and the temperature, which are checked without rows too
template <typename Args> const char* shape_problem(const Args* p) {
    if (const char* why = rows_problem(p->rows, p->V)) return why;
    if (!temperature_ok(p->temperature)) return "need a temperature in [1e-6, 1e6]";
    if (!elem_ok(p->elem)) return "unknown element type";
    return nullptr;
}

template <typename Args> TokenArgs token_args(const Args* p, void* grad, int64_t ld_grad) {
    TokenArgs a{};
    a.rows = p->rows;
    a.V = p->V;
    a.logits = p->logits;
    a.elem = p->elem;
    a.ld = p->ld;
    a.tokens = p->tokens;
    a.inv_tau = 1.0 / p->temperature;
    a.log2_tau = log2_over(p->temperature);
    a.grad = grad;
    a.ld_grad = ld_grad;
    return a;
}

bool all_aligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (!aligned(p, 4)) return false;
    return true;
}

const char* kMisaligned = "buffer not aligned to its elements";

// null, or why the tensors cannot be taken
const char* tensors_problem(int64_t count, const void* const* data, const int64_t* sizes, const int32_t* elems,
                            int32_t order, const float* norm) {
    if (count < 0 || count > HBSJD_GRAD_MAX_TENSORS) return "need 0 to 65536 tensors";
    if (order != 2 && order != 0) return "order must be 2, or 0 for the largest magnitude";
    if (!norm) return "NULL buffer";
    if (!aligned(norm, 4)) return kMisaligned;
    if (count && (!data || !sizes || !elems)) return "NULL array";
    for (int64_t i = 0; i < count; ++i) {
        if (!elem_ok(elems[i])) return "unknown element type";
        if (sizes[i] < 0 || sizes[i] >= (int64_t)1 << 40) return "need sizes in [0, 2^40)";
        if (sizes[i] && !data[i]) return "NULL buffer";
        if (!aligned(data[i], elem_size(elems[i]))) return kMisaligned;
    }
    return nullptr;
}

// whether a written tensor shares memory with another tensor (itself as input aside)
bool written_overlap(int64_t count, void* const* data, const int64_t* sizes, const int32_t* elems,
                     void* const* out) {
    struct Range {
        uintptr_t begin, end;
        bool written;
    };
    std::vector<Range> v;
    v.reserve(2 * count);
    bool ascending = true;
    auto add = [&](const void* p, int64_t i, bool written) {
        const uintptr_t at = (uintptr_t)p;
        ascending = ascending && (v.empty() || v.back().begin <= at);
        v.push_back({at, at + (uintptr_t)sizes[i] * elem_size(elems[i]), written});
    };
    for (int64_t i = 0; i < count; ++i)
        if (sizes[i]) add(out[i], i, true);
    for (int64_t i = 0; i < count; ++i)
        if (sizes[i] && data[i] != out[i]) add(data[i], i, false);
    if (!ascending)
        std::sort(v.begin(), v.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t any = 0, written = 0;
    for (const Range& r : v) {
        if (r.begin < (r.written ? any : written)) return true;
        any = std::max(any, r.end);
        if (r.written) written = std::max(written, r.end);
    }
    return false;
}

}  // namespace

extern "C" {

uint64_t hbsjd_token_workspace(int64_t rows, int32_t V, int32_t elem) {
    if (rows < 1 || rows_problem(rows, V) || !elem_ok(elem)) return 0;
    return token_workspace(rows, V, elem);
}

uint64_t hbsjd_preference_workspace(int64_t rows, int32_t V, int32_t elem) {
    if (rows < 1 || rows_problem(rows, V) || !elem_ok(elem)) return 0;
    return preference_workspace(rows, V, elem);
}

uint64_t hbsjd_grad_norm_workspace(void) { return grad_norm_workspace(); }

hbsjd_status hbsjd_logprob_rows(const hbsjd_logprob_args* p, float* logprob, float* entropy, void* grad,
                                int64_t ld_grad, void* workspace, uint64_t workspace_bytes, void* stream) {
    try {
        if (!p) return api_fail(HBSJD_EINVAL, "args is NULL");
        if (const char* why = shape_problem(p)) return api_fail(HBSJD_EINVAL, why);
        if (p->rows == 0) return HBSJD_OK;
        if (!logprob && !entropy && !grad) return api_fail(HBSJD_EINVAL, "no output");
        if (grad && !p->logprob_weight && !p->entropy_weight)
            return api_fail(HBSJD_EINVAL, "a gradient without a weight");
        if (const char* why = token_problem(p, grad, ld_grad)) return api_fail(HBSJD_EINVAL, why);
        if (!all_aligned({logprob, entropy, p->logprob_weight, p->entropy_weight}))
            return api_fail(HBSJD_EINVAL, kMisaligned);
        if (const char* why = workspace_problem(workspace, workspace_bytes,
                                                token_workspace(p->rows, p->V, p->elem)))
            return api_fail(HBSJD_EINVAL, why);
        TokenArgs a = token_args(p, grad, ld_grad);
        a.logprob = logprob;
        a.entropy = entropy;
        if (grad) {   // without one the weights change nothing and are not read
            a.logprob_weight = p->logprob_weight;
            a.entropy_weight = p->entropy_weight;
        }
        token_rows(a, workspace, (hipStream_t)stream);
        return launched("logprob_rows");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_logprob_rows");
    }
}

hbsjd_status hbsjd_policy_rows(const hbsjd_policy_args* p, float* loss, float* logprob, float* entropy,
                               void* grad, int64_t ld_grad, void* workspace, uint64_t workspace_bytes,
                               void* stream) {
    try {
        if (!p) return api_fail(HBSJD_EINVAL, "args is NULL");
        if (const char* why = shape_problem(p)) return api_fail(HBSJD_EINVAL, why);
        if (!(p->clip_low >= 0.f && p->clip_low <= 1.f)) return api_fail(HBSJD_EINVAL, "need clip_low in [0, 1]");
        if (!weight_ok(p->clip_high)) return api_fail(HBSJD_EINVAL, "need clip_high in [0, 1e6]");
        if (!weight_ok(p->kl_weight) || !weight_ok(p->entropy_weight))
            return api_fail(HBSJD_EINVAL, "need weights in [0, 1e6]");
        if (p->rows == 0) return HBSJD_OK;
        if (!loss && !logprob && !entropy && !grad) return api_fail(HBSJD_EINVAL, "no output");
        if (const char* why = token_problem(p, grad, ld_grad)) return api_fail(HBSJD_EINVAL, why);
        if (!p->advantage) return api_fail(HBSJD_EINVAL, "NULL buffer");
        if (p->kl_weight > 0.f && !p->ref_logprob)
            return api_fail(HBSJD_EINVAL, "the KL term needs ref_logprob");
        if (!all_aligned({loss, logprob, entropy, p->advantage, p->old_logprob, p->ref_logprob, p->row_weight}))
            return api_fail(HBSJD_EINVAL, kMisaligned);
        if (const char* why = workspace_problem(workspace, workspace_bytes,
                                                token_workspace(p->rows, p->V, p->elem)))
            return api_fail(HBSJD_EINVAL, why);
        TokenArgs a = token_args(p, grad, ld_grad);
        a.logprob = logprob;
        a.entropy = entropy;
        a.advantage = p->advantage;
        a.old_logprob = p->old_logprob;
        a.ref_logprob = p->ref_logprob;
        a.low = 1.0 - (double)p->clip_low;
        a.high = 1.0 + (double)p->clip_high;
        a.kl = p->kl_weight;
        a.bonus = p->entropy_weight;
        a.weight = p->row_weight;
        a.loss = loss;
        token_rows(a, workspace, (hipStream_t)stream);
        return launched("policy_rows");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_policy_rows");
    }
}

hbsjd_status hbsjd_preference_rows(const hbsjd_preference_args* p, float* loss, float* log_ratio, void* grad,
                                   int64_t ld_grad, void* workspace, uint64_t workspace_bytes,
                                   void* stream) {
    try {
        if (!p) return api_fail(HBSJD_EINVAL, "args is NULL");
        if (const char* why = shape_problem(p)) return api_fail(HBSJD_EINVAL, why);
        if (p->pairs < 0 || p->pairs >= 1 << 30) return api_fail(HBSJD_EINVAL, "need 0 <= pairs < 2^30");
        if (p->form != HBSJD_PREFERENCE_SIGMOID && p->form != HBSJD_PREFERENCE_HINGE &&
            p->form != HBSJD_PREFERENCE_SQUARE)
            return api_fail(HBSJD_EINVAL, "unknown form of the loss");
        if (!(p->beta >= 1e-6f && p->beta <= 1e6f)) return api_fail(HBSJD_EINVAL, "need beta in [1e-6, 1e6]");
        if (!(p->smoothing >= 0.f && p->smoothing < 1.f))
            return api_fail(HBSJD_EINVAL, "need smoothing in [0, 1)");
        if (p->smoothing > 0.f && p->form != HBSJD_PREFERENCE_SIGMOID)
            return api_fail(HBSJD_EINVAL, "smoothing is the sigmoid form's");
        if (!std::isfinite(p->margin)) return api_fail(HBSJD_EINVAL, "need a finite margin");
        if (!p->first && (p->pairs ? p->rows % (2 * p->pairs) : p->rows))
            return api_fail(HBSJD_EINVAL, "without first the rows have to be a multiple of 2 pairs");
        if (p->rows == 0 && p->pairs == 0) return HBSJD_OK;
        // (without pairs the outputs have no entries, and an empty tensor no address)
        if (p->pairs && !loss && !log_ratio && !grad) return api_fail(HBSJD_EINVAL, "no output");
        if (p->rows)
            if (const char* why = token_problem(p, grad, ld_grad)) return api_fail(HBSJD_EINVAL, why);
        if (!all_aligned({loss, log_ratio, p->first, p->ref_logprob, p->pair_weight}))
            return api_fail(HBSJD_EINVAL, kMisaligned);
        const uint64_t need = p->rows ? preference_workspace(p->rows, p->V, p->elem) : 0;
        if (const char* why = workspace_problem(workspace, workspace_bytes, need))
            return api_fail(HBSJD_EINVAL, why);
        if (p->pairs == 0 && !grad) return HBSJD_OK;
        const TokenArgs a = token_args(p, grad, ld_grad);
        const PreferenceArgs q{p->pairs, p->first, p->ref_logprob, p->form, p->mean != 0, p->beta, p->smoothing,
                               p->margin, p->pair_weight, loss, log_ratio};
        preference_rows(a, q, workspace, (hipStream_t)stream);
        return launched("preference_rows");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_preference_rows");
    }
}

hbsjd_status hbsjd_grad_norm(int64_t count, const void* const* data, const int64_t* sizes, const int32_t* elems,
                             int32_t order, float* norm, void* workspace, uint64_t workspace_bytes,
                             void* stream) {
    try {
        if (const char* why = tensors_problem(count, data, sizes, elems, order, norm))
            return api_fail(HBSJD_EINVAL, why);
        if (const char* why = workspace_problem(workspace, workspace_bytes, grad_norm_workspace()))
            return api_fail(HBSJD_EINVAL, why);
        const GradArgs a{count, data, sizes, elems, order, nullptr, 0.f, norm};
        if (!grad_norm(a, workspace, (hipStream_t)stream)) return api_fail(HBSJD_EINVAL, "sizes out of range");
        return launched("grad_norm");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_grad_norm");
    }
}

hbsjd_status hbsjd_clip_grads(int64_t count, void* const* data, const int64_t* sizes, const int32_t* elems,
                              int32_t order, float limit, void* const* out, float* norm, void* workspace,
                              uint64_t workspace_bytes, void* stream) {
    try {
        if (const char* why = tensors_problem(count, data, sizes, elems, order, norm))
            return api_fail(HBSJD_EINVAL, why);
        if (!(limit >= 0.f)) return api_fail(HBSJD_EINVAL, "need a limit of 0 or more");
        if (!out) out = data;
        for (int64_t i = 0; i < count; ++i) {
            if (sizes[i] && !out[i]) return api_fail(HBSJD_EINVAL, "NULL buffer");
            if (!aligned(out[i], elem_size(elems[i]))) return api_fail(HBSJD_EINVAL, kMisaligned);
        }
        if (written_overlap(count, data, sizes, elems, out))
            return api_fail(HBSJD_EINVAL, "a tensor that is written overlaps another");
        if (const char* why = workspace_problem(workspace, workspace_bytes, grad_norm_workspace()))
            return api_fail(HBSJD_EINVAL, why);
        const GradArgs a{count, data, sizes, elems, order, out, limit, norm};
        if (!grad_norm(a, workspace, (hipStream_t)stream)) return api_fail(HBSJD_EINVAL, "sizes out of range");
        return launched("clip_grads");
    } catch (...) {
        return api_fail(HBSJD_EINTERNAL, "unexpected host exception in hbsjd_clip_grads");
    }
}

}  // extern "C"
