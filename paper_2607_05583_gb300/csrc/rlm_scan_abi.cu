// rlm_scan_abi.cu -- the extern "C" entry points of the gated linear recurrence:
// host-side argument checks and dispatch (kernels in rlm_scan.cu).
#include <initializer_list>
#include <numeric>

#include "rlm_check.h"

using namespace rlm;

namespace {

rlm_status check_shape(int64_t B, int64_t L, int64_t D, const char *name) {
    if (B < 1 || L < 1)
        return fail(RLM_ERR_INVALID_ARG, "%s has B=%lld L=%lld (need >= 1)", name, (long long)B, (long long)L);
    if (D < 8 || D % 8 != 0)
        return fail(RLM_ERR_INVALID_ARG, "%s has D=%lld (need D >= 8 and D %% 8 == 0)", name, (long long)D);
    if (B > 65535) return fail(RLM_ERR_UNSUPPORTED, "%s has B=%lld > 65535", name, (long long)B);
    if (L > (int64_t)1 << 24) return fail(RLM_ERR_UNSUPPORTED, "%s has L=%lld > 2^24", name, (long long)L);
    if (D > 1 << 20) return fail(RLM_ERR_UNSUPPORTED, "%s has D=%lld > 2^20", name, (long long)D);
    return RLM_OK;
}

// A field argument; strides of an extent of 1 are set to those of a dense field.
rlm_status check_field(const rlm_strided *t, const char *name, rlm_strided *out) {
    if (!t) return fail(RLM_ERR_INVALID_ARG, "%s is NULL", name);
    if (!t->ptr) return fail(RLM_ERR_INVALID_ARG, "%s->ptr is NULL", name);
    if (!aligned16(t->ptr)) return fail(RLM_ERR_INVALID_ARG, "%s->ptr is not 16-byte aligned", name);
    if (t->dtype != RLM_F32 && t->dtype != RLM_BF16)
        return fail(RLM_ERR_INVALID_ARG, "%s->dtype %d is not RLM_F32 or RLM_BF16", name, (int)t->dtype);
    rlm_status s = check_shape(t->B, t->L, t->D, name);
    if (s != RLM_OK) return s;
    *out = *t;
    if (t->L == 1) out->stride_l = t->D;
    if (t->B == 1) out->stride_b = t->L * out->stride_l;
    const int64_t per16 = 16 / (int64_t)elem_size(t->dtype);
    // (No field reaches over 2^44 elements; that every extent below does not pass 64 bits.)
    const int64_t most = (int64_t)1 << 44;
    if (out->stride_l < 0 || out->stride_l > most / t->L || out->stride_l % per16 != 0)
        return fail(RLM_ERR_INVALID_ARG, "%s has a stride of %lld elements (need a multiple of 16 bytes, >= 0)", name,
                    (long long)out->stride_l);
    if (out->stride_b < 0 || out->stride_b > most / t->B || out->stride_b % per16 != 0)
        return fail(RLM_ERR_INVALID_ARG, "%s has a stride of %lld elements (need a multiple of 16 bytes, >= 0)", name,
                    (long long)out->stride_b);
    return RLM_OK;
}

rlm_status check_like(const rlm_strided *t, const rlm_strided &x, const char *name, rlm_strided *out) {
    rlm_status s = check_field(t, name, out);
    if (s != RLM_OK) return s;
    if (out->B != x.B || out->L != x.L || out->D != x.D || out->dtype != x.dtype)
        return fail(RLM_ERR_INVALID_ARG, "%s must have x's shape and dtype", name);
    return RLM_OK;
}

// Rows (b, t) of an output must not overlap one another.
rlm_status check_rows(const rlm_strided &t, const char *name) {
    const bool in_l = t.L == 1 || t.stride_l >= t.D, in_b = t.B == 1 || t.stride_b >= t.D;
    const bool nested = t.B == 1 || t.L == 1 || t.stride_b >= (t.L - 1) * t.stride_l + t.D ||
                        t.stride_l >= (t.B - 1) * t.stride_b + t.D;
    if (in_l && in_b && nested) return RLM_OK;
    return fail(RLM_ERR_INVALID_ARG, "%s has overlapping rows (strides %lld, %lld)", name, (long long)t.stride_b,
                (long long)t.stride_l);
}

size_t extent_bytes(const rlm_strided &t) {
    return (size_t)((t.B - 1) * t.stride_b + (t.L - 1) * t.stride_l + t.D) * elem_size(t.dtype);
}

// Whether two fields may touch the same bytes.  Fields whose address ranges cross are
// apart only as column ranges of one wider tensor, batch or time first: equal strides, whose
// common divisor all rows are multiples of apart, and columns that do not meet within it.
bool fields_overlap(const rlm_strided &a, const rlm_strided &b) {
    if (!overlap(a.ptr, extent_bytes(a), b.ptr, extent_bytes(b))) return false;
    if (a.dtype != b.dtype || a.B != b.B || a.L != b.L || (a.L > 1 && a.stride_l != b.stride_l) ||
        (a.B > 1 && a.stride_b != b.stride_b))
        return true;
    const int64_t ea = (int64_t)elem_size(a.dtype);
    const int64_t pitch = std::gcd(a.L > 1 ? a.stride_l : 0, a.B > 1 ? a.stride_b : 0) * ea;
    if (pitch == 0) return true;
    int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.ptr) - reinterpret_cast<uintptr_t>(a.ptr)) % pitch;
    if (d < 0) d += pitch;
    return !(d >= a.D * ea && d + b.D * ea <= pitch);
}

rlm_status check_state(const float *p, const char *name) {
    if (p && !aligned16(p)) return fail(RLM_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return RLM_OK;
}

rlm_status check_lengths(const int32_t *p) {
    if (p && (reinterpret_cast<uintptr_t>(p) & 3u) != 0)
        return fail(RLM_ERR_INVALID_ARG, "lengths is not 4-byte aligned");
    return RLM_OK;
}

struct Region {
    const void *p;
    size_t n;
    const char *name;
};

// Dense buffers of a call against its fields.
rlm_status check_apart(std::initializer_list<Region> outs, std::initializer_list<const rlm_strided *> fields) {
    for (const Region &r : outs) {
        if (!r.p) continue;
        for (const rlm_strided *f : fields)
            if (overlap(r.p, r.n, f->ptr, extent_bytes(*f)))
                return fail(RLM_ERR_INVALID_ARG, "%s overlaps a field of the call", r.name);
    }
    return RLM_OK;
}

}  // namespace

extern "C" {

size_t rlm_scan_saved_size(int64_t B, int64_t L, int D) {
    if (check_shape(B, L, D, "shape") != RLM_OK) return 0;
    return (size_t)B * (size_t)((L + RLM_SCAN_CHUNK - 1) / RLM_SCAN_CHUNK) * (size_t)D * sizeof(float);
}

rlm_status rlm_scan_prefill(const rlm_strided *x_, const rlm_strided *g_, int leak, const float *state_in,
                            const rlm_strided *y_, float *state_out, float *saved, const int32_t *lengths,
                            const rlm_launch *ln) {
    rlm_status s;
    rlm_strided x, g, y;
    if ((s = check_field(x_, "x", &x)) != RLM_OK) return s;
    if ((s = check_like(g_, x, "g", &g)) != RLM_OK) return s;
    if ((s = check_like(y_, x, "y", &y)) != RLM_OK) return s;
    if ((s = check_rows(y, "y")) != RLM_OK) return s;
    if (fields_overlap(x, y) || fields_overlap(g, y)) return fail(RLM_ERR_INVALID_ARG, "y overlaps x or g");
    if ((s = check_state(state_in, "state_in")) != RLM_OK || (s = check_state(state_out, "state_out")) != RLM_OK ||
        (s = check_state(saved, "saved")) != RLM_OK || (s = check_lengths(lengths)) != RLM_OK)
        return s;
    const size_t sb = (size_t)x.B * x.D * sizeof(float), vb = rlm_scan_saved_size(x.B, x.L, (int)x.D);
    if ((s = check_apart({{state_out, sb, "state_out"}, {saved, vb, "saved"}}, {&x, &g, &y})) != RLM_OK) return s;
    if ((s = check_apart({{state_in, sb, "state_in"}}, {&y})) != RLM_OK) return s;
    if (state_in && state_out && state_in != state_out && overlap(state_in, sb, state_out, sb))
        return fail(RLM_ERR_INVALID_ARG, "state_in and state_out overlap without being the same buffer");
    if (saved && ((state_in && overlap(saved, vb, state_in, sb)) || (state_out && overlap(saved, vb, state_out, sb))))
        return fail(RLM_ERR_INVALID_ARG, "saved overlaps state_in or state_out");
    if (!ln) return fail(RLM_ERR_INVALID_ARG, "launch is NULL");
    const cudaError_t e = scan_forward(x, g, y, leak != 0, state_in, state_out, saved, lengths,
                                       static_cast<cudaStream_t>(ln->stream));
    if (e != cudaSuccess) return cuda_fail(e, "rlm_scan_prefill launch");
    return RLM_OK;
}

rlm_status rlm_scan_backward(const rlm_strided *dy_, const rlm_strided *x_, const rlm_strided *g_, const float *saved,
                             int leak, const float *d_state_out, const rlm_strided *dx_, const rlm_strided *dg_,
                             float *d_state_in, const int32_t *lengths, const rlm_launch *ln) {
    rlm_status s;
    rlm_strided dy, x, g, dx, dg;
    if ((s = check_field(x_, "x", &x)) != RLM_OK) return s;
    if ((s = check_like(g_, x, "g", &g)) != RLM_OK) return s;
    if ((s = check_like(dy_, x, "dy", &dy)) != RLM_OK) return s;
    if ((s = check_like(dx_, x, "dx", &dx)) != RLM_OK) return s;
    if ((s = check_like(dg_, x, "dg", &dg)) != RLM_OK) return s;
    if ((s = check_rows(dx, "dx")) != RLM_OK || (s = check_rows(dg, "dg")) != RLM_OK) return s;
    for (const rlm_strided *o : {&dx, &dg})
        for (const rlm_strided *i : {&x, &g, &dy})
            if (fields_overlap(*o, *i)) return fail(RLM_ERR_INVALID_ARG, "dx or dg overlaps x, g or dy");
    if (fields_overlap(dx, dg)) return fail(RLM_ERR_INVALID_ARG, "dx and dg overlap");
    if (!saved) return fail(RLM_ERR_INVALID_ARG, "saved is NULL");
    if ((s = check_state(d_state_in, "d_state_in")) != RLM_OK ||
        (s = check_state(d_state_out, "d_state_out")) != RLM_OK || (s = check_state(saved, "saved")) != RLM_OK ||
        (s = check_lengths(lengths)) != RLM_OK)
        return s;
    const size_t sb = (size_t)x.B * x.D * sizeof(float), vb = rlm_scan_saved_size(x.B, x.L, (int)x.D);
    if ((s = check_apart({{d_state_in, sb, "d_state_in"}}, {&x, &g, &dy, &dx, &dg})) != RLM_OK) return s;
    if ((s = check_apart({{saved, vb, "saved"}, {d_state_out, sb, "d_state_out"}}, {&dx, &dg})) != RLM_OK) return s;
    if (d_state_in && overlap(d_state_in, sb, saved, vb))
        return fail(RLM_ERR_INVALID_ARG, "d_state_in overlaps saved");
    if (d_state_in && d_state_out && d_state_in != d_state_out && overlap(d_state_in, sb, d_state_out, sb))
        return fail(RLM_ERR_INVALID_ARG, "d_state_in and d_state_out overlap without being the same buffer");
    if (!ln) return fail(RLM_ERR_INVALID_ARG, "launch is NULL");
    const cudaError_t e = scan_backward(dy, x, g, saved, leak != 0, d_state_out, dx, dg, d_state_in, lengths,
                                        static_cast<cudaStream_t>(ln->stream));
    if (e != cudaSuccess) return cuda_fail(e, "rlm_scan_backward launch");
    return RLM_OK;
}

rlm_status rlm_scan_decode(const rlm_strided *x_, const rlm_strided *g_, int leak, float *state, const rlm_strided *y_,
                           const rlm_launch *ln) {
    rlm_status s;
    rlm_strided x, g, y;
    if ((s = check_field(x_, "x_t", &x)) != RLM_OK) return s;
    if (x.L != 1) return fail(RLM_ERR_INVALID_ARG, "x_t must have L == 1 (got %lld)", (long long)x.L);
    if ((s = check_like(g_, x, "g_t", &g)) != RLM_OK) return s;
    if ((s = check_like(y_, x, "y_t", &y)) != RLM_OK) return s;
    if ((s = check_rows(y, "y_t")) != RLM_OK) return s;
    if (fields_overlap(x, y) || fields_overlap(g, y)) return fail(RLM_ERR_INVALID_ARG, "y_t overlaps x_t or g_t");
    if (!state) return fail(RLM_ERR_INVALID_ARG, "state is NULL");
    if ((s = check_state(state, "state")) != RLM_OK) return s;
    if ((s = check_apart({{state, (size_t)x.B * x.D * sizeof(float), "state"}}, {&x, &g, &y})) != RLM_OK) return s;
    if (!ln) return fail(RLM_ERR_INVALID_ARG, "launch is NULL");
    const cudaError_t e = scan_step(x, g, y, leak != 0, state, static_cast<cudaStream_t>(ln->stream));
    if (e != cudaSuccess) return cuda_fail(e, "rlm_scan_decode launch");
    return RLM_OK;
}

}  // extern "C"
