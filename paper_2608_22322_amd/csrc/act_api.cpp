// C ABI of the 8-bit activation operators: argument checks on the host before any HIP call, workspace layout, launches
// on the caller's stream. See include/al.h for the contract of each entry point.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "../../include/al.h"
#include "act_internal.hpp"

namespace {

__attribute__((format(printf, 2, 3))) al_status fail(al_status s, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    return al::api_fail(s, msg);
}

al_status launched(hipError_t e, const char* who) {
    return e == hipSuccess ? AL_OK : fail(AL_EHIP, "%s launch: %s", who, hipGetErrorString(e));
}

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

uintptr_t at(const void* p) { return reinterpret_cast<uintptr_t>(p); }

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

bool valid_block(int32_t b) { return b == 32 || b == 64 || b == 128; }

// Most rows, most columns (so that column numbers past the last chunk a kernel looks at stay in 32 bits).
constexpr int64_t kMostRows = (int64_t(1) << 31) - 1, kMostCols = kMostRows - 8192;

al_status check_dtype(int32_t d, const char* who, const char* name) {
    if (d != AL_DTYPE_F32 && d != AL_DTYPE_BF16) return fail(AL_EINVAL, "%s: %s %d", who, name, d);
    return AL_OK;
}

al_status check_shape(int64_t rows, int64_t cols, const char* who) {
    if (rows < 0 || cols < 0) return fail(AL_EINVAL, "%s: negative shape", who);
    if (rows > kMostRows || cols > kMostCols) return fail(AL_EUNSUPPORTED, "%s: %lld x %lld is too large", who, (long long)rows, (long long)cols);
    return AL_OK;
}

// A matrix operand; `need` false: NULL is fine. The row pitch of a single row says nothing, and is taken as cols.
al_status check_mat(const void* p, int64_t* ld, int64_t rows, int64_t cols, int32_t dtype, bool need, const char* who, const char* name) {
    if (!p) return need ? fail(AL_EINVAL, "%s: %s is NULL", who, name) : AL_OK;
    if (rows <= 1)
        *ld = cols;
    else if (*ld < cols)
        return fail(AL_EINVAL, "%s: %s has row pitch %lld < %lld columns", who, name, (long long)*ld, (long long)cols);
    else if (*ld > (int64_t(1) << 48) / rows)
        return fail(AL_EUNSUPPORTED, "%s: %s spans too much memory", who, name);
    if (at(p) & (dtype == AL_DTYPE_BF16 ? 1u : 3u)) return fail(AL_EALIGN, "%s: %s is not aligned to its type", who, name);
    return AL_OK;
}

al_status check_vec(const void* p, int32_t dtype, const char* who, const char* name) {
    if (at(p) & (dtype == AL_DTYPE_BF16 ? 1u : 3u)) return fail(AL_EALIGN, "%s: %s is not aligned to its type", who, name);
    return AL_OK;
}

al_status check_code(const void* codes, const void* exps, const char* who, const char* name) {
    if (!codes || !exps) return fail(AL_EINVAL, "%s: %s codes or exponents are NULL", who, name);
    if ((at(codes) | at(exps)) & 15u) return fail(AL_EALIGN, "%s: %s codes or exponents not 16-byte aligned", who, name);
    return AL_OK;
}

al_status check_block(int32_t block, const char* who) {
    if (!valid_block(block)) return fail(AL_EINVAL, "%s: block %d must be 32, 64 or 128", who, block);
    return AL_OK;
}

al_status check_ws(const void* ws, size_t have, size_t need, const char* who) {
    if (need == 0) return AL_OK;
    if (!ws) return fail(AL_EWORKSPACE, "%s: workspace is NULL (need %zu bytes)", who, need);
    if (have < need) return fail(AL_EWORKSPACE, "%s: workspace %zu bytes < %zu needed", who, have, need);
    if (at(ws) & 255u) return fail(AL_EALIGN, "%s: workspace not 256-byte aligned", who);
    return AL_OK;
}

al::Mat mat(const void* p, int64_t ld) { return {const_cast<void*>(p), ld}; }

al::Code code(const void* c, const void* e) {
    return {static_cast<int8_t*>(const_cast<void*>(c)), static_cast<uint8_t*>(const_cast<void*>(e))};
}

al_status check_kind(int32_t kind, const char* who) {
    if (kind != AL_NORM_LAYER && kind != AL_NORM_RMS) return fail(AL_EINVAL, "%s: kind %d", who, kind);
    return AL_OK;
}

// The grids of the products hold these (2^38 outputs are 2^26 of the smallest tiles, and more than the memory holds).
al_status check_product(int64_t out, int64_t in, const char* who) {
    if (out >= (int64_t(1) << 22) || in >= (int64_t(1) << 29))
        return fail(AL_EUNSUPPORTED, "%s: %lld out_features (below 2^22) or %lld in_features (below 2^29)", who, (long long)out, (long long)in);
    if (out * in > (int64_t(1) << 38)) return fail(AL_EUNSUPPORTED, "%s: %lld x %lld weights are too many", who, (long long)out, (long long)in);
    return AL_OK;
}

size_t norm_ws(int32_t kind, int64_t rows, int64_t cols) {
    const bool layer = kind == AL_NORM_LAYER;
    return align256((size_t)al::norm_backward_parts(rows, cols) * cols * 4 * (layer ? 2 : 1));
}

}  // namespace

#define AL_TRY(x)                              \
    do {                                       \
        const al_status st_ = (x);             \
        if (st_ != AL_OK) return st_;          \
    } while (0)

extern "C" {

int64_t al_act_code_bytes(int64_t rows, int64_t cols, int32_t block) {
    if (rows < 0 || cols < 0 || rows > kMostRows || cols > kMostCols || !valid_block(block)) return -1;
    return rows * ((cols + block - 1) / block) * block;
}

int64_t al_act_exp_bytes(int64_t rows, int64_t cols, int32_t block) {
    if (rows < 0 || cols < 0 || rows > kMostRows || cols > kMostCols || !valid_block(block)) return -1;
    return rows * ((cols + block - 1) / block);
}

al_status al_act_quantize(int32_t dtype, const void* x, int64_t ld, int64_t rows, int64_t cols, int32_t block,
                          void* codes, void* exps, void* stream) {
    const char* const who = "al_act_quantize";
    al::api_clear();
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(rows, cols, who));
    AL_TRY(check_block(block, who));
    if (rows == 0 || cols == 0) return AL_OK;
    AL_TRY(check_mat(x, &ld, rows, cols, dtype, true, who, "x"));
    AL_TRY(check_code(codes, exps, who, "x"));
    return launched(al::launch_act_quantize(dtype, mat(x, ld), al::code_shape(rows, cols, block), code(codes, exps), as_stream(stream)), who);
}

al_status al_act_dequantize(const void* codes, const void* exps, int64_t rows, int64_t cols, int32_t block,
                            int32_t dtype, void* out, int64_t ld, void* stream) {
    const char* const who = "al_act_dequantize";
    al::api_clear();
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(rows, cols, who));
    AL_TRY(check_block(block, who));
    if (rows == 0 || cols == 0) return AL_OK;
    AL_TRY(check_mat(out, &ld, rows, cols, dtype, true, who, "out"));
    AL_TRY(check_code(codes, exps, who, "x"));
    return launched(al::launch_act_dequantize(dtype, code(codes, exps), al::code_shape(rows, cols, block), mat(out, ld), as_stream(stream)), who);
}

al_status al_norm_forward(int32_t kind, int32_t dtype, const void* x, int64_t ldx, int64_t rows, int64_t cols,
                          double eps, const float* gamma, const float* beta, void* y, int64_t ldy, float* mean,
                          float* rstd, int32_t block, void* codes, void* exps, void* stream) {
    const char* const who = "al_norm_forward";
    al::api_clear();
    const bool save = codes || exps;
    AL_TRY(check_kind(kind, who));
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(rows, cols, who));
    if (!std::isfinite(eps) || eps < 0) return fail(AL_EINVAL, "%s: eps must be finite and >= 0", who);
    if (save) AL_TRY(check_block(block, who));
    if (kind == AL_NORM_RMS && (beta || mean)) return fail(AL_EINVAL, "%s: beta and mean must be NULL for an RMS norm", who);
    if (rows == 0 || cols == 0) return AL_OK;
    AL_TRY(check_mat(x, &ldx, rows, cols, dtype, true, who, "x"));
    AL_TRY(check_mat(y, &ldy, rows, cols, dtype, true, who, "y"));
    if (x == y && ldx != ldy) return fail(AL_EINVAL, "%s: y may be x with the same row pitch only", who);
    AL_TRY(check_vec(gamma, AL_DTYPE_F32, who, "gamma"));
    AL_TRY(check_vec(beta, AL_DTYPE_F32, who, "beta"));
    AL_TRY(check_vec(mean, AL_DTYPE_F32, who, "mean"));
    AL_TRY(check_vec(rstd, AL_DTYPE_F32, who, "rstd"));
    if (save) AL_TRY(check_code(codes, exps, who, "xhat"));
    al::NormForward a;
    std::memset(&a, 0, sizeof(a));
    a.x = mat(x, ldx);
    a.y = mat(y, ldy);
    a.s = al::code_shape(rows, cols, save ? block : 32);
    if (!save) a.s.pitch = (int32_t)((cols + 7) / 8 * 8);
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.c = code(codes, exps);
    a.eps = (float)eps;
    return launched(al::launch_norm_forward(dtype, kind == AL_NORM_LAYER, a, as_stream(stream)), who);
}

al_status al_norm_backward_workspace_bytes(int32_t kind, int32_t dtype, int64_t rows, int64_t cols, size_t* bytes) {
    const char* const who = "al_norm_backward_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    AL_TRY(check_kind(kind, who));
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(rows, cols, who));
    *bytes = norm_ws(kind, rows, cols);
    return AL_OK;
}

al_status al_norm_backward(int32_t kind, int32_t dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                           const float* mean, const float* rstd, int32_t block, const void* codes, const void* exps,
                           int64_t rows, int64_t cols, const float* gamma, const void* add, int64_t ldadd, void* dx,
                           int64_t lddx, int32_t grad_dtype, void* dgamma, void* dbeta, void* ws, size_t ws_bytes,
                           void* stream) {
    const char* const who = "al_norm_backward";
    al::api_clear();
    const bool layer = kind == AL_NORM_LAYER, coded = codes || exps;
    AL_TRY(check_kind(kind, who));
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_dtype(grad_dtype, who, "grad_dtype"));
    AL_TRY(check_shape(rows, cols, who));
    if (coded) AL_TRY(check_block(block, who));
    if (dbeta && !layer) return fail(AL_EINVAL, "%s: dbeta must be NULL for an RMS norm", who);
    if (mean && (coded || !layer)) return fail(AL_EINVAL, "%s: mean goes with x and a layer norm only", who);
    if (x && coded) return fail(AL_EINVAL, "%s: either x or its code", who);
    AL_TRY(check_vec(gamma, AL_DTYPE_F32, who, "gamma"));
    AL_TRY(check_vec(mean, AL_DTYPE_F32, who, "mean"));
    AL_TRY(check_vec(rstd, AL_DTYPE_F32, who, "rstd"));
    AL_TRY(check_vec(dgamma, grad_dtype, who, "dgamma"));
    AL_TRY(check_vec(dbeta, grad_dtype, who, "dbeta"));
    if (cols == 0) return AL_OK;
    if (rows > 0) {
        AL_TRY(check_mat(dy, &lddy, rows, cols, dtype, true, who, "dy"));
        if (coded)
            AL_TRY(check_code(codes, exps, who, "xhat"));
        else
            AL_TRY(check_mat(x, &ldx, rows, cols, dtype, true, who, "x"));
        AL_TRY(check_mat(add, &ldadd, rows, cols, dtype, false, who, "add"));
        AL_TRY(check_mat(dx, &lddx, rows, cols, dtype, true, who, "dx"));
        if (add == dx && ldadd != lddx) return fail(AL_EINVAL, "%s: dx may be add with the same row pitch only", who);
        if (dx == dy || dx == x) return fail(AL_EINVAL, "%s: dx must not be dy or x", who);
        if (!rstd || (layer && !coded && !mean)) return fail(AL_EINVAL, "%s: mean or rstd is NULL", who);
    }
    const bool weights = dgamma || dbeta;
    if (weights) AL_TRY(check_ws(ws, ws_bytes, norm_ws(kind, rows, cols), who));
    al::NormBackward a;
    std::memset(&a, 0, sizeof(a));
    a.dy = mat(dy, lddy);
    a.x = mat(x, ldx);
    a.add = mat(add, ldadd);
    a.dx = mat(dx, lddx);
    a.s = al::code_shape(rows, cols, coded ? block : 32);
    a.mean = mean;
    a.rstd = rstd;
    a.gamma = gamma;
    a.c = code(codes, exps);
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.part = weights ? static_cast<float*>(ws) : nullptr;
    a.parts = al::norm_backward_parts(rows, cols);
    a.grad_bf16 = grad_dtype == AL_DTYPE_BF16;
    return launched(al::launch_norm_backward(dtype, layer, grad_dtype, a, as_stream(stream)), who);
}

al_status al_swiglu_forward(int32_t dtype, const void* gate, int64_t ldgate, const void* up, int64_t ldup,
                            int64_t rows, int64_t cols, void* h, int64_t ldh, int32_t block, void* gate_codes,
                            void* gate_exps, void* up_codes, void* up_exps, void* stream) {
    const char* const who = "al_swiglu_forward";
    al::api_clear();
    const bool save = gate_codes || gate_exps || up_codes || up_exps;
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(rows, cols, who));
    if (save) AL_TRY(check_block(block, who));
    if (rows == 0 || cols == 0) return AL_OK;
    AL_TRY(check_mat(gate, &ldgate, rows, cols, dtype, true, who, "gate"));
    AL_TRY(check_mat(up, &ldup, rows, cols, dtype, true, who, "up"));
    AL_TRY(check_mat(h, &ldh, rows, cols, dtype, true, who, "h"));
    if (save) {
        AL_TRY(check_code(gate_codes, gate_exps, who, "gate"));
        AL_TRY(check_code(up_codes, up_exps, who, "up"));
    }
    al::CodeShape s = al::code_shape(rows, cols, save ? block : 32);
    if (!save) s.pitch = (int32_t)((cols + 7) / 8 * 8);
    return launched(al::launch_swiglu_forward(dtype, mat(gate, ldgate), mat(up, ldup), mat(h, ldh), s, code(gate_codes, gate_exps),
                                              code(up_codes, up_exps), as_stream(stream)), who);
}

al_status al_swiglu_backward(int32_t dtype, const void* dh, int64_t lddh, int64_t rows, int64_t cols, int32_t block,
                             const void* gate_codes, const void* gate_exps, const void* up_codes,
                             const void* up_exps, void* dgate, int64_t lddgate, void* dup, int64_t lddup,
                             void* h_codes, void* h_exps, void* stream) {
    const char* const who = "al_swiglu_backward";
    al::api_clear();
    const bool save = h_codes || h_exps;
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(rows, cols, who));
    AL_TRY(check_block(block, who));
    if (rows == 0 || cols == 0) return AL_OK;
    AL_TRY(check_mat(dh, &lddh, rows, cols, dtype, true, who, "dh"));
    AL_TRY(check_code(gate_codes, gate_exps, who, "gate"));
    AL_TRY(check_code(up_codes, up_exps, who, "up"));
    AL_TRY(check_mat(dgate, &lddgate, rows, cols, dtype, true, who, "dgate"));
    AL_TRY(check_mat(dup, &lddup, rows, cols, dtype, true, who, "dup"));
    if (save) AL_TRY(check_code(h_codes, h_exps, who, "h"));
    return launched(al::launch_swiglu_backward(dtype, mat(dh, lddh), code(gate_codes, gate_exps), code(up_codes, up_exps),
                                               al::code_shape(rows, cols, block), mat(dgate, lddgate), mat(dup, lddup),
                                               code(h_codes, h_exps), as_stream(stream)), who);
}

al_status al_linear_wgrad_workspace_bytes(int32_t dtype, int64_t tokens, int64_t out_features, int64_t in_features,
                                          size_t* bytes) {
    const char* const who = "al_linear_wgrad_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(tokens, in_features, who));
    AL_TRY(check_shape(tokens, out_features, who));
    AL_TRY(check_product(out_features, in_features, who));
    const al::WgradPlan p = al::wgrad_plan(dtype, tokens, out_features, in_features);
    *bytes = align256(p.part_bytes) + align256(p.bsum_bytes);
    return AL_OK;
}

al_status al_diag_wgrad_plan(int32_t dtype, int64_t tokens, int64_t out_features, int64_t in_features, int32_t plan[4]) {
    const char* const who = "al_diag_wgrad_plan";
    al::api_clear();
    if (!plan) return fail(AL_EINVAL, "%s: plan is NULL", who);
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_shape(tokens, in_features, who));
    AL_TRY(check_shape(tokens, out_features, who));
    AL_TRY(check_product(out_features, in_features, who));
    const al::WgradPlan p = al::wgrad_plan(dtype, tokens, out_features, in_features);
    plan[0] = p.tile;
    plan[1] = p.splits;
    plan[2] = p.bparts;
    plan[3] = p.beside;
    return AL_OK;
}

al_status al_linear_wgrad(int32_t dtype, const void* dy, int64_t lddy, const void* codes, const void* exps,
                          int32_t block, int64_t tokens, int64_t out_features, int64_t in_features,
                          const float* gamma, const float* beta, int32_t grad_dtype, const void* base, void* dw,
                          void* dbias, void* ws, size_t ws_bytes, void* stream) {
    const char* const who = "al_linear_wgrad";
    al::api_clear();
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_dtype(grad_dtype, who, "grad_dtype"));
    AL_TRY(check_shape(tokens, in_features, who));
    AL_TRY(check_shape(tokens, out_features, who));
    AL_TRY(check_block(block, who));
    AL_TRY(check_product(out_features, in_features, who));
    if (out_features == 0) return AL_OK;
    if (in_features > 0) {
        if (!dw) return fail(AL_EINVAL, "%s: dw is NULL", who);
        if ((at(dw) | at(base)) & 15u) return fail(AL_EALIGN, "%s: dw or base not 16-byte aligned", who);
    }
    if (tokens > 0) {
        AL_TRY(check_mat(dy, &lddy, tokens, out_features, dtype, true, who, "dy"));
        if (in_features > 0) AL_TRY(check_code(codes, exps, who, "xhat"));
    }
    AL_TRY(check_vec(gamma, AL_DTYPE_F32, who, "gamma"));
    AL_TRY(check_vec(beta, AL_DTYPE_F32, who, "beta"));
    AL_TRY(check_vec(dbias, grad_dtype, who, "dbias"));
    const al::WgradPlan p = al::wgrad_plan(dtype, tokens, out_features, in_features);
    AL_TRY(check_ws(ws, ws_bytes, align256(p.part_bytes) + align256(p.bsum_bytes), who));
    al::Wgrad a;
    std::memset(&a, 0, sizeof(a));
    a.dy = mat(dy, lddy);
    a.s = al::code_shape(tokens, in_features, block);
    a.out = out_features;
    a.c = code(codes, exps);
    a.gamma = gamma;
    a.beta = beta;
    a.base = base;
    a.dw = dw;
    a.dbias = dbias;
    a.tile = p.tile;
    a.splits = p.splits;
    a.bparts = p.bparts;
    a.beside = p.beside;
    a.part = static_cast<float*>(ws);
    if (beta || dbias) a.bsum = reinterpret_cast<float*>(static_cast<char*>(ws) + align256(p.part_bytes));
    return launched(al::launch_wgrad(dtype, grad_dtype, a, as_stream(stream)), who);
}

}  // extern "C"
