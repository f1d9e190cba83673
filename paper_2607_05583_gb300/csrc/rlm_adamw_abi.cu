// rlm_adamw_abi.cu -- the extern "C" entry point of the optimizer step: host-side
// argument checks and dispatch (kernels in rlm_adamw.cu).
#include <cmath>

#include "rlm_check.h"

using namespace rlm;

namespace {

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

rlm_status check_entry(const rlm_adamw_tensor &t, int i, rlm_dtype param, rlm_dtype grad, int bits, bool master) {
    if (t.n < 1) return fail(RLM_ERR_INVALID_ARG, "tensors[%d].n=%lld (need >= 1)", i, (long long)t.n);
    if (t.n > (int64_t)1 << 40) return fail(RLM_ERR_UNSUPPORTED, "tensors[%d].n=%lld > 2^40", i, (long long)t.n);
    if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq)
        return fail(RLM_ERR_INVALID_ARG, "tensors[%d] has a NULL param, grad, exp_avg or exp_avg_sq", i);
    if ((t.master != nullptr) != master)
        return fail(RLM_ERR_INVALID_ARG, "tensors[%d]: either every tensor of a call has a master copy or none", i);
    if (!aligned(t.param, elem_size(param)) || !aligned(t.grad, elem_size(grad)) || !aligned(t.master, 4) ||
        (bits == 32 && (!aligned(t.exp_avg, 4) || !aligned(t.exp_avg_sq, 4))))
        return fail(RLM_ERR_INVALID_ARG, "tensors[%d] has a buffer that is not aligned to its elements", i);
    if (bits == 8) {
        if (!t.exp_avg_scale || !t.exp_avg_sq_scale)
            return fail(RLM_ERR_INVALID_ARG, "tensors[%d] has 8-bit moments without scales", i);
        if (!aligned(t.exp_avg_scale, 4) || !aligned(t.exp_avg_sq_scale, 4))
            return fail(RLM_ERR_INVALID_ARG, "tensors[%d] has scales that are not 4-byte aligned", i);
    }
    // The buffers of one tensor against each other (other tensors' are the caller's to keep apart).
    const size_t n = (size_t)t.n, ms = bits == 8 ? 1 : 4, sc = bits == 8 ? (n + RLM_ADAMW_BLOCK - 1) / RLM_ADAMW_BLOCK * 4 : 0;
    const void *p[] = {t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.master, t.exp_avg_scale, t.exp_avg_sq_scale};
    const size_t bytes[] = {n * elem_size(param), n * elem_size(grad), n * ms, n * ms, master ? n * 4 : 0, sc, sc};
    for (int a = 0; a < 7; ++a)
        for (int b = a + 1; b < 7; ++b)
            if (bytes[a] && bytes[b] && overlap(p[a], bytes[a], p[b], bytes[b]))
                return fail(RLM_ERR_INVALID_ARG, "tensors[%d] has overlapping buffers", i);
    return RLM_OK;
}

}  // namespace

extern "C" {

rlm_status rlm_adamw_step(const rlm_adamw_tensor *tensors, int count, rlm_dtype param, rlm_dtype grad, int bits,
                          const rlm_adamw_hyper *h, const float *grad_scale, const rlm_launch *ln) {
    if (!tensors || count < 1) return fail(RLM_ERR_INVALID_ARG, "tensors is NULL or count=%d < 1", count);
    if ((param != RLM_F32 && param != RLM_BF16) || (grad != RLM_F32 && grad != RLM_BF16))
        return fail(RLM_ERR_INVALID_ARG, "param or grad dtype is not RLM_F32 or RLM_BF16");
    const bool draw = bits == (8 | RLM_ADAMW_DRAW);
    if (draw) bits = 8;
    if (bits != 8 && bits != 32) return fail(RLM_ERR_INVALID_ARG, "bits=%d (need 8, 8 | RLM_ADAMW_DRAW or 32)", bits);
    if (!h) return fail(RLM_ERR_INVALID_ARG, "hyper is NULL");
    // Written so that NaN fails.
    if (!(h->lr >= 0 && std::isfinite(h->lr) && h->eps >= 0 && std::isfinite(h->eps) && h->weight_decay >= 0 &&
          std::isfinite(h->weight_decay)))
        return fail(RLM_ERR_INVALID_ARG, "lr, eps and weight_decay must be finite and >= 0");
    if (!(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1))
        return fail(RLM_ERR_INVALID_ARG, "beta1 and beta2 must lie in [0, 1)");
    if (h->step < 1) return fail(RLM_ERR_INVALID_ARG, "step=%lld (need >= 1)", (long long)h->step);
    if (!aligned(grad_scale, 4)) return fail(RLM_ERR_INVALID_ARG, "grad_scale is not 4-byte aligned");
    const bool master = tensors[0].master != nullptr;
    if (master && param != RLM_BF16) return fail(RLM_ERR_INVALID_ARG, "a master copy goes with RLM_BF16 weights");
    for (int i = 0; i < count; ++i) {
        const rlm_status s = check_entry(tensors[i], i, param, grad, bits, master);
        if (s != RLM_OK) return s;
    }
    if (!ln) return fail(RLM_ERR_INVALID_ARG, "launch is NULL");
    const cudaError_t e = adamw_step(tensors, count, param, grad, master, bits, draw, *h, grad_scale,
                                     static_cast<cudaStream_t>(ln->stream));
    if (e != cudaSuccess) return cuda_fail(e, "rlm_adamw_step launch");
    return RLM_OK;
}

}  // extern "C"
