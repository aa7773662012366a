// C ABI of layer norm, rotary positions and dense attention over packed sequences: argument checks and launch plans.
// All checks run before the first launch; nothing here allocates, frees or synchronises.
#include <math.h>

#include "psa_internal.h"

namespace psa {

static bool off_by(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
static bool good_dtype(int32_t d) { return d == PSA_F32 || d == PSA_BF16; }

// ---- layer norm
static int check_norm(int64_t rows, int32_t cols, int32_t dtype)
{
    if (!good_dtype(dtype)) return PSA_ERR_DTYPE;
    if (rows < 1 || rows > INT32_MAX || cols < 1 || cols > (1 << 24)) return PSA_ERR_SHAPE;
    return PSA_OK;
}

// ---- heads
// Strides (and limits that keep offsets inside a tile of rows within 31 bits), `out`: rows of an output must not overlap.
int check_heads(const psa_heads_t& t, int64_t unit, int64_t width, size_t align, int64_t batches, int64_t heads, int64_t rows, bool out)
{
    const int64_t stride[3] = {t.batch_stride, t.head_stride, t.row_stride}, count[3] = {batches, heads, rows};
    for (int i = 0; i < 3; ++i) {
        if (stride[i] < 0) return PSA_ERR_ARG;
        if (count[i] > 1 && out && stride[i] < width) return PSA_ERR_ARG;
        // the last element's offset within 62 bits
        if (count[i] > 1 && stride[i] > (INT64_MAX >> 3) / count[i]) return PSA_ERR_ARG;
    }
    if (rows > 1 && t.row_stride > (1 << 22)) return PSA_ERR_ARG;
    for (int i = 0; i < 3; ++i) if (stride[i] % unit != 0 && count[i] > 1) return PSA_ERR_ALIGN;
    if (off_by(t.data, align)) return PSA_ERR_ALIGN;
    return PSA_OK;
}
static int check_heads(const psa_heads_t& t, int dtype, int64_t batches, int64_t heads, int64_t rows, bool out)
{
    return check_heads(t, dtype == PSA_F32 ? 4 : 8, 64, 16, batches, heads, rows, out);
}

// ---- rotary positions
static bool positive(double x) { return x > 0.0 && isfinite(x); }
static int check_rotary(const psa_rotary_t& o)
{
    if (o.dim < 2 || o.dim > 64 || o.dim % 2 != 0) return PSA_ERR_ARG;
    if (o.layout != PSA_ROTARY_HALF && o.layout != PSA_ROTARY_INTERLEAVED) return PSA_ERR_ARG;
    if (o.scaling < PSA_ROTARY_PLAIN || o.scaling > PSA_ROTARY_PARTS) return PSA_ERR_ARG;
    if (!positive(o.base) || o.base < 1.0 || !positive(o.factor) || !positive(o.magnitude)) return PSA_ERR_ARG;
    // (a frequency beyond float64, or a magnitude beyond float32, would make infinities and NaN of every element)
    if (!positive(1.0 / o.factor) || !positive((float)o.magnitude)) return PSA_ERR_ARG;
    if (o.scaling == PSA_ROTARY_BASE && o.dim > 2 && !positive(o.base * pow(o.factor, (double)o.dim / (o.dim - 2)))) return PSA_ERR_ARG;
    if (o.scaling == PSA_ROTARY_PARTS &&
        (!positive(o.original_length) || !isfinite(o.fast_turns) || !isfinite(o.slow_turns) || !(o.fast_turns > o.slow_turns))) return PSA_ERR_ARG;
    return PSA_OK;
}
static void frequencies(const psa_rotary_t& o, double* f)
{
    double base = o.base;
    if (o.scaling == PSA_ROTARY_BASE && o.dim > 2) base *= pow(o.factor, (double)o.dim / (o.dim - 2));
    for (int i = 0; i < o.dim / 2; ++i) {
        const double x = pow(base, -2.0 * i / o.dim);
        if (o.scaling == PSA_ROTARY_LINEAR) {
            f[i] = x / o.factor;
        } else if (o.scaling == PSA_ROTARY_PARTS) {
            const double turns = o.original_length * x / 6.283185307179586477;
            const double s = fmin(fmax((turns - o.slow_turns) / (o.fast_turns - o.slow_turns), 0.0), 1.0);
            f[i] = x * s + x / o.factor * (1.0 - s);
        } else {
            f[i] = x;
        }
    }
}
static int run_rotary(const psa_heads_t* Q, const psa_heads_t* K, int32_t H_kv, const psa_rotary_t* rotary, const int32_t* positions,
                      int64_t positions_stride, int32_t first, const psa_heads_t* Qo, const psa_heads_t* Ko, const psa_shape_t* s,
                      void* stream, bool back)
{
    if (!Q || !Qo || !rotary || !s || !Q->data || !Qo->data || !K != !Ko || (K && (!K->data || !Ko->data))) return PSA_ERR_NULL;
    if (!good_dtype(s->dtype)) return PSA_ERR_DTYPE;
    if (s->B < 1 || s->B > 65535 || s->H < 1 || s->H > 65535 || s->L_K < 1 || s->L_Q != s->L_K || s->D != kD) return PSA_ERR_SHAPE;
    if (K && (H_kv < 1 || H_kv > 65535)) return PSA_ERR_SHAPE;
    if (s->L_K > (1 << 22)) return PSA_ERR_SHAPE;
    int rc = check_rotary(*rotary);
    if (rc != PSA_OK) return rc;
    if (positions) {
        if (positions_stride != 0 && positions_stride < s->L_K) return PSA_ERR_ARG;
        if (off_by(positions, 4)) return PSA_ERR_ALIGN;
    } else if ((int64_t)first + s->L_K > INT32_MAX) {
        return PSA_ERR_ARG;
    }
    const int L = s->L_K;
    if ((rc = check_heads(*Q, s->dtype, s->B, s->H, L, false)) != PSA_OK || (rc = check_heads(*Qo, s->dtype, s->B, s->H, L, true)) != PSA_OK) return rc;
    if (K && ((rc = check_heads(*K, s->dtype, s->B, H_kv, L, false)) != PSA_OK || (rc = check_heads(*Ko, s->dtype, s->B, H_kv, L, true)) != PSA_OK)) return rc;
    double freq[32];
    frequencies(*rotary, freq);
    return launch_rotary(Q, K, H_kv, *rotary, freq, back, positions, positions_stride, first, Qo, Ko, *s, static_cast<hipStream_t>(stream)) == hipSuccess
        ? PSA_OK : PSA_ERR_HIP;
}

// ---- packed attention
constexpr int64_t kMostGroups = (1 << 24) - 1;         // work-groups of 256 threads
static int check_packed(const psa_packed_shape_t* s)
{
    if (!s) return PSA_ERR_NULL;
    if (!good_dtype(s->dtype)) return PSA_ERR_DTYPE;
    if (s->B < 1 || s->H < 1 || s->H_kv < 1 || s->T_q < 1 || s->T_k < 1 || s->D != kD || s->H % s->H_kv != 0) return PSA_ERR_SHAPE;
    if (s->B > (1 << 20) || s->H > 65535 || s->T_q > (1 << 28) || s->T_k > (1 << 28)) return PSA_ERR_SHAPE;
    if ((int64_t)s->T_q * (s->H / s->H_kv) > INT32_MAX - 65536) return PSA_ERR_SHAPE;
    // (the kernels hold scale * log2(e) in float32: 0 there would make NaN of a masked score)
    if ((s->causal != 0 && s->causal != 1) || !(s->scale >= 1e-30) || !(s->scale <= 1e30)) return PSA_ERR_ARG;
    // a launch has fewer than 2^32 threads
    const PackedBwdPlan b = make_packed_bwd_plan(*s);
    if ((int64_t)make_packed_plan(*s).n_tile * s->H_kv > kMostGroups || ((int64_t)b.n_qtile + b.n_ktile) * s->H_kv > kMostGroups) return PSA_ERR_SHAPE;
    return PSA_OK;
}
static int check_offsets(const psa_packed_shape_t& s, const int32_t* qo, const int32_t* ko)
{
    if (!qo != !ko) return PSA_ERR_NULL;
    if (!qo && s.B != 1) return PSA_ERR_NULL;
    if (off_by(qo, 4) || off_by(ko, 4)) return PSA_ERR_ALIGN;
    return PSA_OK;
}
static bool has_data(const psa_heads_t* t) { return t && t->data; }

}  // namespace psa

extern "C" {

int probsparse_layer_norm_fwd(const void* X, const void* gamma, const void* beta, double eps, void* Y, float* mean, float* rstd,
                              int64_t rows, int32_t cols, int32_t dtype, void* stream)
{
    using namespace psa;
    if (!X || !Y || !mean != !rstd) return PSA_ERR_NULL;
    const int rc = check_norm(rows, cols, dtype);
    if (rc != PSA_OK) return rc;
    if (!(eps >= 0.0) || !isfinite((float)eps)) return PSA_ERR_ARG;
    if (off_by(X, 16) || off_by(Y, 16) || off_by(gamma, 16) || off_by(beta, 16) || off_by(mean, 4) || off_by(rstd, 4)) return PSA_ERR_ALIGN;
    return launch_norm_fwd(make_norm_plan(rows, cols, dtype, true), X, gamma, beta, (float)eps, Y, mean, rstd, rows, cols, dtype,
                           static_cast<hipStream_t>(stream)) == hipSuccess ? PSA_OK : PSA_ERR_HIP;
}

size_t probsparse_layer_norm_bwd_workspace_bytes(int64_t rows, int32_t cols, int32_t dtype)
{
    return psa::check_norm(rows, cols, dtype) == PSA_OK ? psa::make_norm_plan(rows, cols, dtype, false).total : 0;
}

int probsparse_layer_norm_bwd(const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd, void* dX,
                              float* dgamma, float* dbeta, int64_t rows, int32_t cols, int32_t dtype, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    using namespace psa;
    if (!dY || !X || !mean || !rstd || !dX || !dgamma != !dbeta || !workspace) return PSA_ERR_NULL;
    const int rc = check_norm(rows, cols, dtype);
    if (rc != PSA_OK) return rc;
    if (off_by(dY, 16) || off_by(X, 16) || off_by(gamma, 16) || off_by(dX, 16) || off_by(mean, 4) || off_by(rstd, 4) ||
        off_by(dgamma, 4) || off_by(dbeta, 4) || off_by(workspace, 256)) return PSA_ERR_ALIGN;
    const NormPlan p = make_norm_plan(rows, cols, dtype, false);
    if (workspace_bytes < p.total) return PSA_ERR_WORKSPACE;
    return launch_norm_bwd(p, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, rows, cols, dtype, workspace,
                           static_cast<hipStream_t>(stream)) == hipSuccess ? PSA_OK : PSA_ERR_HIP;
}

int probsparse_rotary_frequencies(const psa_rotary_t* rotary, double* freq)
{
    if (!rotary || !freq) return PSA_ERR_NULL;
    const int rc = psa::check_rotary(*rotary);
    if (rc == PSA_OK) psa::frequencies(*rotary, freq);
    return rc;
}

int probsparse_rotary_fwd(const psa_heads_t* Q, const psa_heads_t* K, int32_t H_kv, const psa_rotary_t* rotary, const int32_t* positions,
                          int64_t positions_stride, int32_t first, const psa_heads_t* Q_out, const psa_heads_t* K_out,
                          const psa_shape_t* shape, void* stream)
{
    return psa::run_rotary(Q, K, H_kv, rotary, positions, positions_stride, first, Q_out, K_out, shape, stream, false);
}

int probsparse_rotary_bwd(const psa_heads_t* dQ_out, const psa_heads_t* dK_out, int32_t H_kv, const psa_rotary_t* rotary,
                          const int32_t* positions, int64_t positions_stride, int32_t first, const psa_heads_t* dQ, const psa_heads_t* dK,
                          const psa_shape_t* shape, void* stream)
{
    return psa::run_rotary(dQ_out, dK_out, H_kv, rotary, positions, positions_stride, first, dQ, dK, shape, stream, true);
}

size_t dense_attn_packed_workspace_bytes(const psa_packed_shape_t* shape)
{
    return psa::check_packed(shape) == PSA_OK ? psa::make_packed_plan(*shape).total : 0;
}

int dense_attn_packed_fwd(const psa_heads_t* Q, const psa_heads_t* K, const psa_heads_t* V, const int32_t* q_offsets,
                          const int32_t* k_offsets, const psa_heads_t* out, float* lse, const psa_packed_shape_t* shape,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace psa;
    if (!has_data(Q) || !has_data(K) || !has_data(V) || !has_data(out) || !workspace) return PSA_ERR_NULL;
    int rc = check_packed(shape);
    if (rc != PSA_OK) return rc;
    const psa_packed_shape_t& s = *shape;
    if ((rc = check_offsets(s, q_offsets, k_offsets)) != PSA_OK || (rc = check_heads(*Q, s.dtype, 1, s.H, s.T_q, false)) != PSA_OK ||
        (rc = check_heads(*K, s.dtype, 1, s.H_kv, s.T_k, false)) != PSA_OK || (rc = check_heads(*V, s.dtype, 1, s.H_kv, s.T_k, false)) != PSA_OK ||
        (rc = check_heads(*out, s.dtype, 1, s.H, s.T_q, true)) != PSA_OK) return rc;
    if (off_by(lse, 4) || off_by(workspace, 256)) return PSA_ERR_ALIGN;
    const PackedPlan p = make_packed_plan(s);
    if (workspace_bytes < p.total) return PSA_ERR_WORKSPACE;
    return launch_packed(p, s, *Q, *K, *V, q_offsets, k_offsets, *out, lse, workspace, static_cast<hipStream_t>(stream)) == hipSuccess
        ? PSA_OK : PSA_ERR_HIP;
}

size_t dense_attn_packed_bwd_workspace_bytes(const psa_packed_shape_t* shape)
{
    return psa::check_packed(shape) == PSA_OK ? psa::make_packed_bwd_plan(*shape).total : 0;
}

int dense_attn_packed_bwd(const psa_heads_t* Q, const psa_heads_t* K, const psa_heads_t* V, const int32_t* q_offsets,
                          const int32_t* k_offsets, const psa_heads_t* out, const float* lse, const psa_heads_t* dOut, const psa_heads_t* dQ,
                          const psa_heads_t* dK, const psa_heads_t* dV, const psa_packed_shape_t* shape, void* workspace,
                          size_t workspace_bytes, void* stream)
{
    using namespace psa;
    if (!has_data(Q) || !has_data(K) || !has_data(V) || !has_data(out) || !lse || !has_data(dOut) || !has_data(dQ) || !has_data(dK) ||
        !has_data(dV) || !workspace) return PSA_ERR_NULL;
    int rc = check_packed(shape);
    if (rc != PSA_OK) return rc;
    const psa_packed_shape_t& s = *shape;
    if ((rc = check_offsets(s, q_offsets, k_offsets)) != PSA_OK) return rc;
    const struct { const psa_heads_t* t; bool keys, out; } all[] = {{Q, false, false}, {K, true, false}, {V, true, false}, {out, false, false},
                                                                   {dOut, false, false}, {dQ, false, true}, {dK, true, true}, {dV, true, true}};
    for (const auto& a : all)
        if ((rc = check_heads(*a.t, s.dtype, 1, a.keys ? s.H_kv : s.H, a.keys ? s.T_k : s.T_q, a.out)) != PSA_OK) return rc;
    if (off_by(lse, 4) || off_by(workspace, 256)) return PSA_ERR_ALIGN;
    const PackedBwdPlan p = make_packed_bwd_plan(s);
    if (workspace_bytes < p.total) return PSA_ERR_WORKSPACE;
    return launch_packed_bwd(p, s, *Q, *K, *V, q_offsets, k_offsets, *out, lse, *dOut, *dQ, *dK, *dV, workspace,
                             static_cast<hipStream_t>(stream)) == hipSuccess ? PSA_OK : PSA_ERR_HIP;
}

}  // extern "C"
