// rlm_linear_abi.cu -- the extern "C" entry points of the linear layer: host-side
// argument checks and dispatch (kernels in rlm_linear.cu).
#include <initializer_list>

#include "rlm_check.h"

using namespace rlm;

namespace {

rlm_status check_sizes(int64_t R, int64_t K, int64_t N) {
    if (R < 1) return fail(RLM_ERR_INVALID_ARG, "x has %lld rows (need >= 1)", (long long)R);
    if (K < 8 || K % 8 != 0 || N < 8 || N % 8 != 0)
        return fail(RLM_ERR_INVALID_ARG, "K=%lld, N=%lld (need multiples of 8, >= 8)", (long long)K, (long long)N);
    if (R > (int64_t)1 << 24 || K > 1 << 20 || N > 1 << 20)
        return fail(RLM_ERR_UNSUPPORTED, "R=%lld, K=%lld, N=%lld (limits 2^24, 2^20, 2^20)", (long long)R, (long long)K,
                    (long long)N);
    return RLM_OK;
}

bool good_act(int act) { return act >= RLM_ACT_NONE && act <= RLM_ACT_SIGMOID; }

rlm_status check_matrix(const rlm_matrix *m, const char *name) {
    if (!m) return fail(RLM_ERR_INVALID_ARG, "%s is NULL", name);
    if (!m->ptr || !aligned16(m->ptr)) return fail(RLM_ERR_INVALID_ARG, "%s->ptr is NULL or not 16-byte aligned", name);
    if (m->dtype != RLM_F32 && m->dtype != RLM_BF16)
        return fail(RLM_ERR_INVALID_ARG, "%s->dtype %d is not RLM_F32 or RLM_BF16", name, (int)m->dtype);
    const int64_t per16 = 16 / (int64_t)elem_size(m->dtype);
    if (m->ld < m->cols || m->ld % per16 != 0 || m->ld > (int64_t)1 << 32)
        return fail(RLM_ERR_INVALID_ARG, "%s->ld=%lld (need at least its %lld columns, a multiple of 16 bytes)", name,
                    (long long)m->ld, (long long)m->cols);
    return RLM_OK;
}

rlm_status check_as(const rlm_matrix *m, const char *name, int64_t rows, int64_t cols, bool f32_too = false) {
    const rlm_status s = check_matrix(m, name);
    if (s != RLM_OK) return s;
    if (m->rows != rows || m->cols != cols)
        return fail(RLM_ERR_INVALID_ARG, "%s is [%lld][%lld], expected [%lld][%lld]", name, (long long)m->rows,
                    (long long)m->cols, (long long)rows, (long long)cols);
    if (m->dtype != RLM_BF16 && !f32_too) return fail(RLM_ERR_UNSUPPORTED, "%s is not RLM_BF16", name);
    return RLM_OK;
}

rlm_status check_vector(const float *p, const char *name) {
    if (p && !aligned16(p)) return fail(RLM_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return RLM_OK;
}

size_t extent(const rlm_matrix &m) { return (size_t)((m.rows - 1) * m.ld + m.cols) * elem_size(m.dtype); }

// Whether two matrices may touch the same bytes.  Crossing address ranges are apart only
// as column ranges of one wider matrix: equal row pitch in bytes, columns side by side.
bool matrices_overlap(const rlm_matrix &a, const rlm_matrix &b) {
    if (!overlap(a.ptr, extent(a), b.ptr, extent(b))) return false;
    const int64_t ea = (int64_t)elem_size(a.dtype), eb = (int64_t)elem_size(b.dtype), pitch = a.ld * ea;
    if (pitch != b.ld * eb) return true;
    int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.ptr) - reinterpret_cast<uintptr_t>(a.ptr)) % pitch;
    if (d < 0) d += pitch;
    return !(d >= a.cols * ea && d + b.cols * eb <= pitch);
}

struct Named {
    const rlm_matrix *m;
    const char *name;
};
// Every output against every input and the outputs after it.
rlm_status check_apart(std::initializer_list<Named> outs, std::initializer_list<Named> ins) {
    for (const Named *o = outs.begin(); o != outs.end(); ++o) {
        if (!o->m) continue;
        for (const Named &i : ins)
            if (i.m && matrices_overlap(*o->m, *i.m))
                return fail(RLM_ERR_INVALID_ARG, "%s overlaps %s", o->name, i.name);
        for (const Named *q = o + 1; q != outs.end(); ++q)
            if (q->m && matrices_overlap(*o->m, *q->m))
                return fail(RLM_ERR_INVALID_ARG, "%s overlaps %s", o->name, q->name);
    }
    return RLM_OK;
}

rlm_matrix row_of(const float *p, int64_t n) { return {const_cast<float *>(p), RLM_F32, 1, n, n}; }

}  // namespace

extern "C" {

size_t rlm_linear_workspace_size(int64_t R, int64_t K, int64_t N) {
    return check_sizes(R, K, N) == RLM_OK ? linear_ws_bytes(R, K, N) : 0;
}

size_t rlm_linear_backward_workspace_size(int64_t R, int64_t K, int64_t N, rlm_act act) {
    return check_sizes(R, K, N) == RLM_OK && good_act(act) ? linear_backward_ws_bytes(R, K, N, act) : 0;
}

rlm_status rlm_linear(const rlm_matrix *x, const rlm_matrix *w, const float *bias, rlm_act act,
                      const rlm_matrix *residual, const rlm_matrix *pre, const rlm_matrix *y, const rlm_launch *ln) {
    rlm_status s;
    if (!x || !w) return fail(RLM_ERR_INVALID_ARG, "x or w is NULL");
    const int64_t R = x->rows, K = x->cols, N = w->rows;
    if ((s = check_sizes(R, K, N)) != RLM_OK) return s;
    if (!good_act(act)) return fail(RLM_ERR_INVALID_ARG, "act %d is not an rlm_act", (int)act);
    if ((s = check_as(x, "x", R, K)) != RLM_OK || (s = check_as(w, "w", N, K)) != RLM_OK ||
        (s = check_as(y, "y", R, N)) != RLM_OK)
        return s;
    if (residual && (s = check_as(residual, "residual", R, N)) != RLM_OK) return s;
    if (pre && (s = check_as(pre, "pre", R, N)) != RLM_OK) return s;
    if ((s = check_vector(bias, "bias")) != RLM_OK) return s;
    const rlm_matrix b = row_of(bias, N);
    const bool in_place = residual && residual->ptr == y->ptr && (residual->ld == y->ld || R == 1);
    if ((s = check_apart({{y, "y"}, {pre, "pre"}}, {{x, "x"}, {w, "w"}, {bias ? &b : nullptr, "bias"}})) != RLM_OK)
        return s;
    if (residual && ((!in_place && matrices_overlap(*residual, *y)) || (pre && matrices_overlap(*residual, *pre))))
        return fail(RLM_ERR_INVALID_ARG, "residual overlaps y or pre");
    if ((s = check_workspace(ln, linear_ws_bytes(R, K, N))) != RLM_OK) return s;
    const cudaError_t e =
        linear_forward(*x, *w, bias, act, residual, pre, *y, ln->workspace, static_cast<cudaStream_t>(ln->stream));
    if (e != cudaSuccess) return cuda_fail(e, "rlm_linear launch");
    return RLM_OK;
}

rlm_status rlm_linear_backward(const rlm_matrix *dy, const rlm_matrix *x, const rlm_matrix *w, const rlm_matrix *pre,
                               rlm_act act, const rlm_matrix *dx, const rlm_matrix *dw, float *dbias,
                               const rlm_launch *ln) {
    rlm_status s;
    if (!x || !w) return fail(RLM_ERR_INVALID_ARG, "x or w is NULL");
    const int64_t R = x->rows, K = x->cols, N = w->rows;
    if ((s = check_sizes(R, K, N)) != RLM_OK) return s;
    if (!good_act(act)) return fail(RLM_ERR_INVALID_ARG, "act %d is not an rlm_act", (int)act);
    if ((s = check_as(dy, "dy", R, N)) != RLM_OK || (s = check_as(x, "x", R, K)) != RLM_OK ||
        (s = check_as(w, "w", N, K)) != RLM_OK)
        return s;
    if ((pre != nullptr) != (act != RLM_ACT_NONE))
        return fail(RLM_ERR_INVALID_ARG, "pre is needed with an activation, and only then");
    if (pre && (s = check_as(pre, "pre", R, N)) != RLM_OK) return s;
    if (dx && (s = check_as(dx, "dx", R, K)) != RLM_OK) return s;
    if (dw && (s = check_as(dw, "dw", N, K, true)) != RLM_OK) return s;
    if ((s = check_vector(dbias, "dbias")) != RLM_OK) return s;
    if (!dx && !dw && !dbias) return fail(RLM_ERR_INVALID_ARG, "none of dx, dw and dbias is given");
    const rlm_matrix b = row_of(dbias, N);
    if ((s = check_apart({{dx, "dx"}, {dw, "dw"}, {dbias ? &b : nullptr, "dbias"}},
                         {{dy, "dy"}, {x, "x"}, {w, "w"}, {pre, "pre"}})) != RLM_OK)
        return s;
    if ((s = check_workspace(ln, linear_backward_ws_bytes(R, K, N, act))) != RLM_OK) return s;
    const cudaError_t e = linear_backward(*dy, *x, *w, pre, act, dx, dw, dbias, ln->workspace,
                                          static_cast<cudaStream_t>(ln->stream));
    if (e != cudaSuccess) return cuda_fail(e, "rlm_linear_backward launch");
    return RLM_OK;
}

}  // extern "C"
