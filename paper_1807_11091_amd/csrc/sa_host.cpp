// Host-side helpers: error reporting and argument validation.  Every entry
// point validates all of its arguments here before anything is enqueued.
#include "sa_host.h"

#include <cstdio>
#include <cstring>

namespace sa {

static thread_local char g_err[512];

int fail(int code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return code;
}

void clear_error() { g_err[0] = '\0'; }

int check_hip(hipError_t e, const char *what) {
    if (e == hipSuccess) return SA_OK;
    return fail(SA_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

static const int64_t kMaxElems = (int64_t(1) << 31) - 1;

int validate_project(const sa_project_desc &d, int i) {
    if (d.A <= 0 || d.B <= 0 || d.C <= 0 || d.D <= 0)
        return fail(SA_E_ARG, "layer %d: shape [%lld,%lld,%lld,%lld] must be positive", i,
                    (long long)d.A, (long long)d.B, (long long)d.C, (long long)d.D);
    if (d.A > kMaxElems / d.B || d.A * d.B > kMaxElems / (d.C * d.D) || d.C * d.D > kMaxElems)
        return fail(SA_E_ARG, "layer %d: A*B*C*D must be below 2^31", i);
    if (d.groups <= 0 || d.A % d.groups != 0)
        return fail(SA_E_ARG, "layer %d: groups=%d must be >= 1 and divide A=%lld", i, d.groups,
                    (long long)d.A);
    if (d.kind < SA_FILTER || d.kind > SA_ELEMENT)
        return fail(SA_E_ARG, "layer %d: unknown kind %d", i, d.kind);
    int64_t G = n_groups(d);
    if (d.k < 0 || d.k > G)
        return fail(SA_E_ARG, "layer %d: k=%lld outside [0, n_groups=%lld]", i, (long long)d.k,
                    (long long)G);
    if (d.kind != SA_ELEMENT && G > SA_MAX_STRUCT_GROUPS)
        return fail(SA_E_UNSUPPORTED, "layer %d: %lld groups exceed the structured selection limit %d",
                    i, (long long)G, SA_MAX_STRUCT_GROUPS);
    if (!d.W || !d.U || !d.Z || !d.mask || (d.k > 0 && !d.kept_idx))
        return fail(SA_E_ARG, "layer %d: W, U, Z, mask and (for k > 0) kept_idx are required", i);
    if (!aligned(d.W, 16) || !aligned(d.U, 16) || !aligned(d.Z, 16) || (d.G && !aligned(d.G, 16)))
        return fail(SA_E_ALIGN, "layer %d: W, U, Z and G must be 16-byte aligned", i);
    if (d.scores && !aligned(d.scores, 8))
        return fail(SA_E_ALIGN, "layer %d: scores must be 8-byte aligned", i);
    if (d.kept_idx && !aligned(d.kept_idx, 4))
        return fail(SA_E_ALIGN, "layer %d: kept_idx must be 4-byte aligned", i);
    if ((const void *)d.Z == (const void *)d.W || d.Z == d.U)
        return fail(SA_E_ARG, "layer %d: Z must not alias W or U", i);
    if (d.G && ((const void *)d.G == (const void *)d.W || d.G == d.U || d.G == d.Z))
        return fail(SA_E_ARG, "layer %d: G must not alias W, U or Z", i);
    return SA_OK;
}

int validate_dual(const sa_dual_desc &d, int i) {
    if (d.n <= 0 || d.n > kMaxElems)
        return fail(SA_E_ARG, "layer %d: n=%lld must be in [1, 2^31)", i, (long long)d.n);
    if (!d.W || !d.Z || !d.U)
        return fail(SA_E_ARG, "layer %d: W, Z and U are required", i);
    if (!d.update_dual && !d.G)
        return fail(SA_E_ARG, "layer %d: nothing to do (update_dual=0 and G=NULL)", i);
    if (!aligned(d.W, 16) || !aligned(d.Z, 16) || !aligned(d.U, 16) || (d.G && !aligned(d.G, 16)))
        return fail(SA_E_ALIGN, "layer %d: W, Z, U and G must be 16-byte aligned", i);
    return SA_OK;
}

int validate_sgd(const sa_sgd_desc &d, int i) {
    if (d.A <= 0 || d.B <= 0 || d.C <= 0 || d.D <= 0)
        return fail(SA_E_ARG, "layer %d: shape must be positive", i);
    if (d.A > kMaxElems / d.B || d.A * d.B > kMaxElems / (d.C * d.D))
        return fail(SA_E_ARG, "layer %d: A*B*C*D must be below 2^31", i);
    if (d.kind < SA_FILTER || d.kind > SA_ELEMENT) return fail(SA_E_ARG, "layer %d: unknown kind %d", i, d.kind);
    if (!d.W || !d.Gf) return fail(SA_E_ARG, "layer %d: W and Gf are required", i);
    if ((d.Z == nullptr) != (d.U == nullptr)) return fail(SA_E_ARG, "layer %d: give both Z and U or neither", i);
    if (d.Gf == d.W) return fail(SA_E_ARG, "layer %d: Gf must not alias W", i);
    if (!aligned(d.W, 16) || !aligned(d.Gf, 16) || (d.Z && (!aligned(d.Z, 16) || !aligned(d.U, 16))))
        return fail(SA_E_ALIGN, "layer %d: W, Gf, Z and U must be 16-byte aligned", i);
    return SA_OK;
}

int validate_compact(const sa_compact_desc &d) {
    if (d.A <= 0 || d.B <= 0 || d.C <= 0 || d.D <= 0)
        return fail(SA_E_ARG, "compact: shape must be positive");
    if (d.A > kMaxElems / d.B || d.A * d.B > kMaxElems / (d.C * d.D))
        return fail(SA_E_ARG, "compact: A*B*C*D must be below 2^31");
    if (d.groups <= 0 || d.groups > SA_MAX_CONV_GROUPS || d.A % d.groups != 0)
        return fail(SA_E_ARG, "compact: groups=%d must be in [1, %d] and divide A", d.groups,
                    SA_MAX_CONV_GROUPS);
    if (d.C > 255 || d.D > 255)
        return fail(SA_E_UNSUPPORTED, "compact: kernel %lldx%lld larger than 255", (long long)d.C,
                    (long long)d.D);
    if ((int64_t)d.groups * d.B > 32768)
        return fail(SA_E_UNSUPPORTED, "compact: more than 32768 input channels");
    if (!d.Z || !d.Wc || !d.row_idx || !d.col_ch || !d.col_tap || !d.ws)
        return fail(SA_E_ARG, "compact: Z, Wc, row_idx, col_ch, col_tap and ws are required");
    if (d.in_compacted && !d.in_ch_mask)
        return fail(SA_E_ARG, "compact: in_compacted requires in_ch_mask");
    if (!aligned(d.Wc, 16) || !aligned(d.ws, 256) || !aligned(d.row_idx, 4) ||
        !aligned(d.col_ch, 4) || !aligned(d.col_tap, 4) || !aligned(d.Z, 4))
        return fail(SA_E_ALIGN, "compact: Wc must be 16-byte, ws 256-byte, tables 4-byte aligned");
    return SA_OK;
}

int validate_conv(const sa_conv_desc &d) {
    if (!d.sizes)
        return fail(SA_E_ARG, "conv: sizes (from structadmm_compact) is required");
    const sa_compact_sizes &s = *d.sizes;
    if (d.N <= 0 || d.H <= 0 || d.W <= 0 || d.Cx <= 0 || d.C <= 0 || d.D <= 0 || d.stride <= 0 ||
        d.pad < 0)
        return fail(SA_E_ARG, "conv: N, H, W, Cx, C, D, stride must be positive and pad >= 0");
    if (s.groups <= 0 || s.groups > SA_MAX_CONV_GROUPS)
        return fail(SA_E_ARG, "conv: sizes->groups=%d out of range", s.groups);
    int64_t P = ((int64_t)d.H + 2 * d.pad - d.C) / d.stride + 1;
    int64_t Q = ((int64_t)d.W + 2 * d.pad - d.D) / d.stride + 1;
    if (d.H + 2 * d.pad < d.C || d.W + 2 * d.pad < d.D || P <= 0 || Q <= 0)
        return fail(SA_E_ARG, "conv: output would be empty");
    if ((int64_t)d.N * P * Q > kMaxElems || (int64_t)d.N * d.H * d.W > kMaxElems)
        return fail(SA_E_UNSUPPORTED, "conv: N*P*Q and N*H*W must be below 2^31");
    if ((int64_t)d.N * d.H * d.W * d.Cx >= (int64_t(1) << 40))
        return fail(SA_E_UNSUPPORTED, "conv: input too large");
    if (d.C > 255 || d.D > 255)
        return fail(SA_E_UNSUPPORTED, "conv: kernel larger than 255");
    int64_t Cy = 0;
    for (int g = 0; g < s.groups; ++g) {
        if (s.M[g] < 0 || s.K[g] < 0)
            return fail(SA_E_ARG, "conv: negative group size");
        if (s.K[g] > 16384)
            return fail(SA_E_UNSUPPORTED, "conv: K=%d columns exceed 16384", s.K[g]);
        if (s.run[g] > 0 && (int64_t)s.run[g] * d.C * d.D != s.K[g])
            return fail(SA_E_ARG, "conv: run[%d]=%d inconsistent with K=%d", g, s.run[g], s.K[g]);
        if (s.run[g] > 0 && s.run_base[g] + s.run[g] > d.Cx)
            return fail(SA_E_ARG, "conv: channel run of group %d exceeds Cx=%d", g, d.Cx);
        Cy += s.M[g];
    }
    if (Cy <= 0)
        return fail(SA_E_ARG, "conv: no output channels");
    if (d.ldy != 0 && d.ldy < Cy)
        return fail(SA_E_ARG, "conv: ldy=%d is below the %lld output channels", d.ldy, (long long)Cy);
    if (!d.X || !d.Wc || !d.Y || !d.col_ch || !d.col_tap)
        return fail(SA_E_ARG, "conv: X, Wc, col_ch, col_tap and Y are required");
    if (!aligned(d.X, 16) || !aligned(d.Wc, 16) || !aligned(d.Y, 4))
        return fail(SA_E_ALIGN, "conv: X and Wc must be 16-byte aligned, Y 4-byte aligned");
    return SA_OK;
}

int check_workspace(const char *who, const void *ws, size_t have, size_t need) {
    if (need == 0) return SA_OK;
    if (!ws || have < need)
        return fail(SA_E_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? have : (size_t)0);
    if (!aligned(ws, 256)) return fail(SA_E_ALIGN, "%s: the workspace must be 256-byte aligned", who);
    return SA_OK;
}

namespace {

size_t type_bytes(int32_t type) { return type == SA_F32 ? 4 : 2; }

// A matrix argument: its pitch, its presence (where it has elements) and the
// alignment of an element.
int check_matrix(const char *who, const char *name, const void *p, bool required, int64_t rows, int64_t cols, int64_t ld,
                 int32_t type, bool pointers) {
    if (!p && !required) return SA_OK;  // left out
    if (ld < cols || ld > SA_MAX_LD)
        return fail(ld < cols ? SA_E_ARG : SA_E_UNSUPPORTED, "%s: the pitch %lld of %s must be in [%lld, %d]", who,
                    (long long)ld, name, (long long)cols, SA_MAX_LD);
    if (pointers && required && !p && rows > 0 && cols > 0) return fail(SA_E_ARG, "%s: %s is required", who, name);
    if (p && !aligned(p, type_bytes(type)))
        return fail(SA_E_ALIGN, "%s: %s must be aligned to its elements", who, name);
    return SA_OK;
}

int check_vector(const char *who, const char *name, const float *p) {
    return p && !aligned(p, 4) ? fail(SA_E_ALIGN, "%s: %s must be 4-byte aligned", who, name) : SA_OK;
}

int check_product(const char *who, int64_t M, int64_t N, int64_t K, int32_t type, int32_t out_type, int32_t act) {
    if (M < 0 || N < 0 || K < 0 || M > kMaxElems || N > SA_MAX_LD || K > SA_MAX_LD)
        return fail(M < 0 || N < 0 || K < 0 ? SA_E_ARG : SA_E_UNSUPPORTED,
                    "%s: M=%lld must be in [0, 2^31), N=%lld and K=%lld in [0, %d]", who, (long long)M, (long long)N,
                    (long long)K, SA_MAX_LD);
    if (type != SA_BF16 && type != SA_F16)
        return fail(type == SA_F32 ? SA_E_UNSUPPORTED : SA_E_ARG, "%s: type %d must be SA_BF16 or SA_F16", who, type);
    if (out_type != type && out_type != SA_F32)
        return fail(SA_E_ARG, "%s: the result's type %d must be the operands' or SA_F32", who, out_type);
    if (act < SA_ACT_NONE || act > SA_ACT_GELU_TANH) return fail(SA_E_ARG, "%s: unknown activation %d", who, act);
    return SA_OK;
}

int check_norm(const char *who, int64_t rows, int64_t cols, int32_t type) {
    if (rows < 0 || rows > kMaxElems || cols < 1)
        return fail(SA_E_ARG, "%s: rows=%lld must be in [0, 2^31) and cols=%lld positive", who, (long long)rows,
                    (long long)cols);
    if (type != SA_BF16 && type != SA_F16 && type != SA_F32) return fail(SA_E_ARG, "%s: unknown type %d", who, type);
    return SA_OK;
}

// an output that is an input: refused unless `same_place`
int check_alias(const char *who, const char *names, const void *out, const void *in, bool same_place = false) {
    if (out && out == in && !same_place) return fail(SA_E_ARG, "%s: %s must not be the same memory", who, names);
    return SA_OK;
}

#define SA_TRY(expr)                    \
    do {                                \
        if (int rc_ = (expr)) return rc_; \
    } while (0)

int check_linear(const sa_linear_desc &d, bool ptrs) {
    const char *w = "linear_fwd";
    SA_TRY(check_product(w, d.M, d.N, d.K, d.type, d.out_type, d.act));
    SA_TRY(check_matrix(w, "X", d.X, true, d.M, d.K, d.ldx, d.type, ptrs));
    SA_TRY(check_matrix(w, "W", d.W, true, d.N, d.K, d.ldw, d.type, ptrs));
    SA_TRY(check_matrix(w, "R", d.R, false, d.M, d.N, d.ldr, d.out_type, ptrs));
    SA_TRY(check_matrix(w, "Y", d.Y, true, d.M, d.N, d.ldy, d.out_type, ptrs));
    SA_TRY(check_matrix(w, "Z", d.Z, false, d.M, d.N, d.ldz, d.type, ptrs));
    SA_TRY(check_vector(w, "bias", d.bias));
    if (!ptrs) return SA_OK;
    SA_TRY(check_alias(w, "Y and X", d.Y, d.X));
    SA_TRY(check_alias(w, "Y and W", d.Y, d.W));
    SA_TRY(check_alias(w, "Y and R with another pitch", d.Y, d.R, d.ldy == d.ldr));
    SA_TRY(check_alias(w, "Z and Y", d.Z, d.Y));
    SA_TRY(check_alias(w, "Z and R", d.Z, d.R));
    SA_TRY(check_alias(w, "Z and X", d.Z, d.X));
    return check_alias(w, "Z and W", d.Z, d.W);
}

int check_linear_bwd(const sa_linear_bwd_desc &d, bool ptrs) {
    const char *w = "linear_bwd";
    SA_TRY(check_product(w, d.M, d.N, d.K, d.type, d.dw_type, d.act));
    SA_TRY(check_matrix(w, "dY", d.dY, true, d.M, d.N, d.lddy, d.type, ptrs));
    SA_TRY(check_matrix(w, "Z", d.Z, d.act != SA_ACT_NONE, d.M, d.N, d.ldz, d.type, ptrs));
    SA_TRY(check_matrix(w, "X", d.X, d.dW != nullptr, d.M, d.K, d.ldx, d.type, ptrs));
    SA_TRY(check_matrix(w, "W", d.W, d.dX != nullptr, d.N, d.K, d.ldw, d.type, ptrs));
    SA_TRY(check_matrix(w, "dX", d.dX, false, d.M, d.K, d.lddx, d.type, ptrs));
    SA_TRY(check_matrix(w, "dW", d.dW, false, d.N, d.K, d.lddw, d.dw_type, ptrs));
    SA_TRY(check_vector(w, "dbias", d.dbias));
    if (!ptrs) return SA_OK;
    if (!d.dX && !d.dW && !d.dbias && d.M > 0 && d.N > 0 && d.K > 0)
        return fail(SA_E_ARG, "%s: nothing to do (dX, dW and dbias are NULL)", w);
    const void *in[] = {d.dY, d.Z, d.X, d.W};
    for (const void *p : in) {
        SA_TRY(check_alias(w, "dX and an input", d.dX, p));
        SA_TRY(check_alias(w, "dW and an input", d.dW, p));
    }
    return check_alias(w, "dX and dW", d.dX, d.dW);
}

int check_glu(const sa_glu_desc &d, bool ptrs) {
    const char *w = "glu_fwd";
    SA_TRY(check_product(w, d.M, d.N, d.K, d.type, d.type, d.act));
    SA_TRY(check_matrix(w, "X", d.X, true, d.M, d.K, d.ldx, d.type, ptrs));
    SA_TRY(check_matrix(w, "Wg", d.Wg, true, d.N, d.K, d.ldw, d.type, ptrs));
    SA_TRY(check_matrix(w, "Wu", d.Wu, true, d.N, d.K, d.ldw, d.type, ptrs));
    SA_TRY(check_matrix(w, "H", d.H, true, d.M, d.N, d.ldh, d.type, ptrs));
    SA_TRY(check_matrix(w, "G", d.G, false, d.M, d.N, d.ldgu, d.type, ptrs));
    SA_TRY(check_matrix(w, "U", d.U, false, d.M, d.N, d.ldgu, d.type, ptrs));
    SA_TRY(check_vector(w, "bg", d.bg));
    SA_TRY(check_vector(w, "bu", d.bu));
    if (!ptrs) return SA_OK;
    if ((d.G == nullptr) != (d.U == nullptr)) return fail(SA_E_ARG, "%s: give both G and U or neither", w);
    const void *in[] = {d.X, d.Wg, d.Wu};
    for (const void *p : in) {
        SA_TRY(check_alias(w, "H and an input", d.H, p));
        SA_TRY(check_alias(w, "G and an input", d.G, p));
        SA_TRY(check_alias(w, "U and an input", d.U, p));
    }
    SA_TRY(check_alias(w, "G and U", d.G, d.U));
    SA_TRY(check_alias(w, "H and G", d.H, d.G));
    return check_alias(w, "H and U", d.H, d.U);
}

int check_glu_bwd(const sa_glu_bwd_desc &d, bool ptrs) {
    const char *w = "glu_bwd";
    SA_TRY(check_product(w, d.M, d.N, d.K, d.type, d.dw_type, d.act));
    SA_TRY(check_matrix(w, "dH", d.dH, true, d.M, d.N, d.lddh, d.type, ptrs));
    SA_TRY(check_matrix(w, "G", d.G, true, d.M, d.N, d.ldgu, d.type, ptrs));
    SA_TRY(check_matrix(w, "U", d.U, true, d.M, d.N, d.ldgu, d.type, ptrs));
    SA_TRY(check_matrix(w, "X", d.X, d.dWg || d.dWu, d.M, d.K, d.ldx, d.type, ptrs));
    SA_TRY(check_matrix(w, "Wg", d.Wg, d.dX != nullptr, d.N, d.K, d.ldw, d.type, ptrs));
    SA_TRY(check_matrix(w, "Wu", d.Wu, d.dX != nullptr, d.N, d.K, d.ldw, d.type, ptrs));
    SA_TRY(check_matrix(w, "dX", d.dX, false, d.M, d.K, d.lddx, d.type, ptrs));
    SA_TRY(check_matrix(w, "dWg", d.dWg, false, d.N, d.K, d.lddw, d.dw_type, ptrs));
    SA_TRY(check_matrix(w, "dWu", d.dWu, false, d.N, d.K, d.lddw, d.dw_type, ptrs));
    SA_TRY(check_vector(w, "dbg", d.dbg));
    SA_TRY(check_vector(w, "dbu", d.dbu));
    if ((d.dWg == nullptr) != (d.dWu == nullptr)) return fail(SA_E_ARG, "%s: give both dWg and dWu or neither", w);
    if (!ptrs) return SA_OK;
    if (!d.dX && !d.dWg && !d.dbg && !d.dbu && d.M > 0 && d.N > 0 && d.K > 0)
        return fail(SA_E_ARG, "%s: nothing to do (every output is NULL)", w);
    const void *in[] = {d.dH, d.G, d.U, d.X, d.Wg, d.Wu};
    for (const void *p : in) {
        SA_TRY(check_alias(w, "dX and an input", d.dX, p));
        SA_TRY(check_alias(w, "dWg and an input", d.dWg, p));
        SA_TRY(check_alias(w, "dWu and an input", d.dWu, p));
    }
    SA_TRY(check_alias(w, "dWg and dWu", d.dWg, d.dWu));
    SA_TRY(check_alias(w, "dX and dWg", d.dX, d.dWg));
    return check_alias(w, "dX and dWu", d.dX, d.dWu);
}

int check_norm_bwd(const sa_layer_norm_bwd_desc &d, bool ptrs) {
    const char *w = "layer_norm_bwd";
    SA_TRY(check_norm(w, d.rows, d.cols, d.type));
    SA_TRY(check_matrix(w, "dY", d.dY, true, d.rows, d.cols, d.lddy, d.type, ptrs));
    SA_TRY(check_matrix(w, "X", d.X, true, d.rows, d.cols, d.ldx, d.type, ptrs));
    SA_TRY(check_matrix(w, "dR", d.dR, false, d.rows, d.cols, d.lddr, d.type, ptrs));
    SA_TRY(check_matrix(w, "dX", d.dX, false, d.rows, d.cols, d.lddx, d.type, ptrs));
    SA_TRY(check_vector(w, "mean", d.mean));
    SA_TRY(check_vector(w, "rstd", d.rstd));
    SA_TRY(check_vector(w, "gamma", d.gamma));
    SA_TRY(check_vector(w, "dgamma", d.dgamma));
    SA_TRY(check_vector(w, "dbeta", d.dbeta));
    if (!ptrs) return SA_OK;
    if (d.rows > 0 && (!d.mean || !d.rstd)) return fail(SA_E_ARG, "%s: mean and rstd are required", w);
    if (!d.dX && !d.dgamma && !d.dbeta && d.rows > 0)
        return fail(SA_E_ARG, "%s: nothing to do (dX, dgamma and dbeta are NULL)", w);
    SA_TRY(check_alias(w, "dX and X", d.dX, d.X));
    SA_TRY(check_alias(w, "dX and dY with another pitch", d.dX, d.dY, d.lddx == d.lddy));
    return check_alias(w, "dX and dR with another pitch", d.dX, d.dR, d.lddx == d.lddr);
}

int64_t blocks_of(int64_t n) { return (n + SA_BLOCK - 1) / SA_BLOCK; }

// An 8-bit matrix of blocks of block_rows rows.  `out`: its scales must not share memory.
int check_matrix8(const char *who, const char *name, const sa_matrix8 &q, bool required, int64_t rows, int64_t cols,
                  int64_t block_rows, bool out, bool pointers) {
    if (!q.codes && !required) return SA_OK;  // left out
    if (q.ld < cols || q.ld > SA_MAX_LD)
        return fail(q.ld < cols ? SA_E_ARG : SA_E_UNSUPPORTED, "%s: the pitch %lld of %s must be in [%lld, %d]", who,
                    (long long)q.ld, name, (long long)cols, SA_MAX_LD);
    if (q.ld % 16) return fail(SA_E_ALIGN, "%s: the pitch %lld of %s must be a multiple of 16", who, (long long)q.ld, name);
    const int64_t nr = block_rows == 1 ? rows : blocks_of(rows), nc = blocks_of(cols);
    if (q.scale_row < 0 || q.scale_col < 0)
        return fail(SA_E_ARG, "%s: the strides of %s's scales must not be negative", who, name);
    if (q.scale_row > SA_MAX_LD || q.scale_col > kMaxElems)
        return fail(SA_E_UNSUPPORTED, "%s: the strides %lld and %lld of %s's scales must be at most %d and 2^31 - 1", who,
                    (long long)q.scale_row, (long long)q.scale_col, name, SA_MAX_LD);
    if (out) {  // rows of block columns or the other way round
        const int64_t r = nr > 1 ? q.scale_row : 1, c = nc > 1 ? q.scale_col : 1;
        const bool by_row = nc <= 1 || (c >= 1 && (nr <= 1 || r >= c * (nc - 1) + 1));
        const bool by_col = nr <= 1 || (r >= 1 && (nc <= 1 || c >= r * (nr - 1) + 1));
        if (r < 1 || c < 1 || !(by_row || by_col))
            return fail(SA_E_ARG, "%s: the strides of %s's scales let blocks share one", who, name);
    }
    if (pointers && rows > 0 && cols > 0 && (!q.codes || !q.scales))
        return fail(SA_E_ARG, "%s: %s is required, codes and scales", who, name);
    if (!aligned(q.codes, 16)) return fail(SA_E_ALIGN, "%s: the codes of %s must be 16-byte aligned", who, name);
    if (!aligned(q.scales, 4)) return fail(SA_E_ALIGN, "%s: the scales of %s must be 4-byte aligned", who, name);
    return SA_OK;
}

// an 8-bit output against an operand or another output
int check_alias8(const char *who, const char *names, const sa_matrix8 &out, const void *in) {
    SA_TRY(check_alias(who, names, out.codes, in));
    return out.codes ? check_alias(who, names, out.scales, in) : SA_OK;
}
int check_alias8(const char *who, const char *names, const sa_matrix8 &out, const sa_matrix8 &in) {
    SA_TRY(check_alias8(who, names, out, in.codes));
    return in.codes ? check_alias8(who, names, out, in.scales) : SA_OK;
}

int check_rms_bwd(const sa_rms_norm_bwd_desc &d, bool ptrs) {
    const char *w = "rms_norm_bwd";
    SA_TRY(check_norm(w, d.rows, d.cols, d.type));
    SA_TRY(check_matrix(w, "dY", d.dY, true, d.rows, d.cols, d.lddy, d.type, ptrs));
    SA_TRY(check_matrix(w, "S", d.S, true, d.rows, d.cols, d.lds, d.type, ptrs));
    SA_TRY(check_matrix(w, "dR", d.dR, false, d.rows, d.cols, d.lddr, d.type, ptrs));
    SA_TRY(check_matrix(w, "dX", d.dX, false, d.rows, d.cols, d.lddx, d.type, ptrs));
    SA_TRY(check_vector(w, "rstd", d.rstd));
    SA_TRY(check_vector(w, "gamma", d.gamma));
    SA_TRY(check_vector(w, "dgamma", d.dgamma));
    if (!ptrs) return SA_OK;
    if (d.rows > 0 && !d.rstd) return fail(SA_E_ARG, "%s: rstd is required", w);
    if (!d.dX && !d.dgamma && d.rows > 0) return fail(SA_E_ARG, "%s: nothing to do (dX and dgamma are NULL)", w);
    SA_TRY(check_alias(w, "dX and S", d.dX, d.S));
    SA_TRY(check_alias(w, "dX and dY with another pitch", d.dX, d.dY, d.lddx == d.lddy));
    return check_alias(w, "dX and dR with another pitch", d.dX, d.dR, d.lddx == d.lddr);
}

int check_linear8(const sa_linear8_desc &d, bool ptrs) {
    const char *w = "linear8_fwd";
    SA_TRY(check_product(w, d.M, d.N, d.K, d.type, d.out_type, d.act));
    if (d.exact != 0 && d.exact != 1) return fail(SA_E_ARG, "%s: exact=%d must be 0 or 1", w, d.exact);
    SA_TRY(check_matrix8(w, "X", d.X, true, d.M, d.K, 1, false, ptrs));
    SA_TRY(check_matrix8(w, "W", d.W, true, d.N, d.K, SA_BLOCK, false, ptrs));
    SA_TRY(check_matrix(w, "R", d.R, false, d.M, d.N, d.ldr, d.out_type, ptrs));
    SA_TRY(check_matrix(w, "Y", d.Y, false, d.M, d.N, d.ldy, d.out_type, ptrs));
    SA_TRY(check_matrix(w, "Z", d.Z, false, d.M, d.N, d.ldz, d.type, ptrs));
    SA_TRY(check_matrix8(w, "Q", d.Q, false, d.M, d.N, 1, true, ptrs));
    SA_TRY(check_vector(w, "bias", d.bias));
    if (!ptrs) return SA_OK;
    if (!d.Y && !d.Q.codes && d.M > 0 && d.N > 0) return fail(SA_E_ARG, "%s: Y or Q is required", w);
    const void *in[] = {d.X.codes, d.X.scales, d.W.codes, d.W.scales};
    for (const void *p : in) {
        SA_TRY(check_alias(w, "Y and an operand", d.Y, p));
        SA_TRY(check_alias(w, "Z and an operand", d.Z, p));
        SA_TRY(check_alias8(w, "Q and an operand", d.Q, p));
    }
    SA_TRY(check_alias(w, "Y and R with another pitch", d.Y, d.R, d.ldy == d.ldr));
    SA_TRY(check_alias(w, "Z and Y", d.Z, d.Y));
    SA_TRY(check_alias(w, "Z and R", d.Z, d.R));
    SA_TRY(check_alias8(w, "Q and Y", d.Q, d.Y));
    SA_TRY(check_alias8(w, "Q and Z", d.Q, d.Z));
    return check_alias8(w, "Q and R", d.Q, d.R);
}

int check_glu8(const sa_glu8_desc &d, bool ptrs) {
    const char *w = "glu8_fwd";
    SA_TRY(check_product(w, d.M, d.N, d.K, d.type, d.type, d.act));
    if (d.exact != 0 && d.exact != 1) return fail(SA_E_ARG, "%s: exact=%d must be 0 or 1", w, d.exact);
    SA_TRY(check_matrix8(w, "X", d.X, true, d.M, d.K, 1, false, ptrs));
    SA_TRY(check_matrix8(w, "Wg", d.Wg, true, d.N, d.K, SA_BLOCK, false, ptrs));
    SA_TRY(check_matrix8(w, "Wu", d.Wu, true, d.N, d.K, SA_BLOCK, false, ptrs));
    if (d.N > 1 && d.Wg.ld != d.Wu.ld) return fail(SA_E_ARG, "%s: Wg and Wu must have one pitch", w);
    if ((d.N > SA_BLOCK && d.Wg.scale_row != d.Wu.scale_row) || (d.K > SA_BLOCK && d.Wg.scale_col != d.Wu.scale_col))
        return fail(SA_E_ARG, "%s: the scales of Wg and Wu must have the same strides", w);
    SA_TRY(check_matrix(w, "H", d.H, false, d.M, d.N, d.ldh, d.type, ptrs));
    SA_TRY(check_matrix(w, "G", d.G, false, d.M, d.N, d.ldgu, d.type, ptrs));
    SA_TRY(check_matrix(w, "U", d.U, false, d.M, d.N, d.ldgu, d.type, ptrs));
    SA_TRY(check_matrix8(w, "Q", d.Q, false, d.M, d.N, 1, true, ptrs));
    SA_TRY(check_vector(w, "bg", d.bg));
    SA_TRY(check_vector(w, "bu", d.bu));
    if ((d.G == nullptr) != (d.U == nullptr)) return fail(SA_E_ARG, "%s: give both G and U or neither", w);
    if (!ptrs) return SA_OK;
    if (!d.H && !d.Q.codes && d.M > 0 && d.N > 0) return fail(SA_E_ARG, "%s: H or Q is required", w);
    const void *in[] = {d.X.codes, d.X.scales, d.Wg.codes, d.Wg.scales, d.Wu.codes, d.Wu.scales};
    for (const void *p : in) {
        SA_TRY(check_alias(w, "H and an operand", d.H, p));
        SA_TRY(check_alias(w, "G and an operand", d.G, p));
        SA_TRY(check_alias(w, "U and an operand", d.U, p));
        SA_TRY(check_alias8(w, "Q and an operand", d.Q, p));
    }
    SA_TRY(check_alias(w, "G and U", d.G, d.U));
    SA_TRY(check_alias(w, "H and G", d.H, d.G));
    SA_TRY(check_alias(w, "H and U", d.H, d.U));
    SA_TRY(check_alias8(w, "Q and H", d.Q, d.H));
    SA_TRY(check_alias8(w, "Q and G", d.Q, d.G));
    return check_alias8(w, "Q and U", d.Q, d.U);
}

}  // namespace

int validate_layer_norm(const sa_layer_norm_desc &d) {
    const char *w = "layer_norm_fwd";
    SA_TRY(check_norm(w, d.rows, d.cols, d.type));
    if (!(d.eps >= 0.0f)) return fail(SA_E_ARG, "%s: eps must be at least 0", w);
    SA_TRY(check_matrix(w, "X", d.X, true, d.rows, d.cols, d.ldx, d.type, true));
    SA_TRY(check_matrix(w, "Y", d.Y, true, d.rows, d.cols, d.ldy, d.type, true));
    SA_TRY(check_vector(w, "gamma", d.gamma));
    SA_TRY(check_vector(w, "beta", d.beta));
    SA_TRY(check_vector(w, "mean", d.mean));
    SA_TRY(check_vector(w, "rstd", d.rstd));
    return check_alias(w, "Y and X with another pitch", d.Y, d.X, d.ldy == d.ldx);
}

int validate_layer_norm_bwd_sizes(const sa_layer_norm_bwd_desc &d) { return check_norm_bwd(d, false); }
int validate_layer_norm_bwd(const sa_layer_norm_bwd_desc &d) { return check_norm_bwd(d, true); }
int validate_linear_sizes(const sa_linear_desc &d) { return check_linear(d, false); }
int validate_linear(const sa_linear_desc &d) { return check_linear(d, true); }
int validate_linear_bwd_sizes(const sa_linear_bwd_desc &d) { return check_linear_bwd(d, false); }
int validate_linear_bwd(const sa_linear_bwd_desc &d) { return check_linear_bwd(d, true); }
int validate_glu_sizes(const sa_glu_desc &d) { return check_glu(d, false); }
int validate_glu(const sa_glu_desc &d) { return check_glu(d, true); }
int validate_glu_bwd_sizes(const sa_glu_bwd_desc &d) { return check_glu_bwd(d, false); }
int validate_glu_bwd(const sa_glu_bwd_desc &d) { return check_glu_bwd(d, true); }
int validate_rms_norm_bwd_sizes(const sa_rms_norm_bwd_desc &d) { return check_rms_bwd(d, false); }
int validate_rms_norm_bwd(const sa_rms_norm_bwd_desc &d) { return check_rms_bwd(d, true); }
int validate_linear8_sizes(const sa_linear8_desc &d) { return check_linear8(d, false); }
int validate_linear8(const sa_linear8_desc &d) { return check_linear8(d, true); }
int validate_glu8_sizes(const sa_glu8_desc &d) { return check_glu8(d, false); }
int validate_glu8(const sa_glu8_desc &d) { return check_glu8(d, true); }

int validate_rms_norm(const sa_rms_norm_desc &d) {
    const char *w = "rms_norm_fwd";
    SA_TRY(check_norm(w, d.rows, d.cols, d.type));
    if (!(d.eps >= 0.0f)) return fail(SA_E_ARG, "%s: eps must be at least 0", w);
    SA_TRY(check_matrix(w, "X", d.X, true, d.rows, d.cols, d.ldx, d.type, true));
    SA_TRY(check_matrix(w, "R", d.R, false, d.rows, d.cols, d.ldr, d.type, true));
    SA_TRY(check_matrix(w, "S", d.S, false, d.rows, d.cols, d.lds, d.type, true));
    SA_TRY(check_matrix(w, "Y", d.Y, false, d.rows, d.cols, d.ldy, d.type, true));
    SA_TRY(check_matrix8(w, "Q", d.Q, false, d.rows, d.cols, 1, true, true));
    SA_TRY(check_vector(w, "gamma", d.gamma));
    SA_TRY(check_vector(w, "rstd", d.rstd));
    if (!d.S && !d.Y && !d.Q.codes && !d.rstd && d.rows > 0)
        return fail(SA_E_ARG, "%s: nothing to do (S, Y, Q and rstd are NULL)", w);
    SA_TRY(check_alias(w, "S and X with another pitch", d.S, d.X, d.lds == d.ldx));
    SA_TRY(check_alias(w, "S and R with another pitch", d.S, d.R, d.lds == d.ldr));
    SA_TRY(check_alias(w, "Y and X with another pitch", d.Y, d.X, d.ldy == d.ldx));
    SA_TRY(check_alias(w, "Y and R with another pitch", d.Y, d.R, d.ldy == d.ldr));
    SA_TRY(check_alias(w, "Y and S", d.Y, d.S));
    const void *other[] = {d.X, d.R, d.S, d.Y};
    for (const void *p : other) SA_TRY(check_alias8(w, "Q and another matrix", d.Q, p));
    return SA_OK;
}

int validate_quantize8(const sa_quantize8_desc &d) {
    const char *w = "quantize8";
    if (d.rows < 0 || d.rows > kMaxElems || d.cols < 0)
        return fail(SA_E_ARG, "%s: rows=%lld must be in [0, 2^31) and cols=%lld at least 0", w, (long long)d.rows,
                    (long long)d.cols);
    if (d.type != SA_BF16 && d.type != SA_F16 && d.type != SA_F32) return fail(SA_E_ARG, "%s: unknown type %d", w, d.type);
    if (d.block_rows != 1 && d.block_rows != SA_BLOCK)
        return fail(SA_E_ARG, "%s: block_rows=%d must be 1 or %d", w, d.block_rows, SA_BLOCK);
    SA_TRY(check_matrix(w, "X", d.X, true, d.rows, d.cols, d.ldx, d.type, true));
    SA_TRY(check_matrix8(w, "Q", d.Q, false, d.rows, d.cols, d.block_rows, true, true));
    SA_TRY(check_matrix8(w, "QT", d.QT, false, d.cols, d.rows, d.block_rows, true, true));
    if (!d.Q.codes && !d.QT.codes && d.rows > 0 && d.cols > 0)
        return fail(SA_E_ARG, "%s: nothing to do (Q and QT are NULL)", w);
    SA_TRY(check_alias8(w, "Q and X", d.Q, d.X));
    SA_TRY(check_alias8(w, "QT and X", d.QT, d.X));
    return check_alias8(w, "Q and QT", d.Q, d.QT);
}

#undef SA_TRY

}  // namespace sa

extern "C" const char *structadmm_last_error(void) { return sa::g_err; }

extern "C" const char *structadmm_version(void) { return "structadmm-gfx950 0.1"; }
