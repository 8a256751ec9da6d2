// C ABI of the orthogonalised updates: argument checks on the host before any HIP call, workspace layout, launches on the caller's stream. See
// include/al.h for the contract of each entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "api_checks.hpp"
#include "ortho_internal.hpp"

namespace {

constexpr int kMostSteps = 64;
constexpr double kMostSigma = 4.0, kMostPoly = 128.0;  // what fp16 holds of X, A and b A + c A A at their scales

// The coefficients, followed over the steps: the largest singular value of X (t = its square) and of b A + c A A.
al_status check_ortho(const al_ortho_cfg& k, const char* who) {
    if (!std::isfinite(k.a) || !std::isfinite(k.b) || !std::isfinite(k.c) || !std::isfinite(k.eps) || k.eps < 0)
        return fail(AL_EINVAL, "%s: coefficients or eps out of range", who);
    if (k.steps < 1 || k.steps > kMostSteps) return fail(AL_EINVAL, "%s: steps %d must be 1 to %d", who, k.steps, kMostSteps);
    if (k.parts != 1 && k.parts != 2) return fail(AL_EINVAL, "%s: parts %d must be 1 or 2", who, k.parts);
    double top = 1.0;
    for (int i = 0; i < k.steps; ++i) {
        const double most = top * top;
        double at[4] = {most, 0, 0, 0};  // ends and turning points of a + b t + c t^2 times sqrt(t), and of b t + c t^2
        int n = 1;
        const auto add = [&](double t) {
            if (t > 0 && t < most) at[n++] = t;
        };
        if (k.c != 0) {
            const double disc = 9 * k.b * k.b - 20 * k.a * k.c;
            if (disc >= 0) {
                add((-3 * k.b + std::sqrt(disc)) / (10 * k.c));
                add((-3 * k.b - std::sqrt(disc)) / (10 * k.c));
            }
        } else if (k.b != 0) {
            add(-k.a / (3 * k.b));
        }
        double next = 0, poly = std::fabs(k.b * most + k.c * most * most);
        if (k.c != 0 && -k.b / (2 * k.c) > 0 && -k.b / (2 * k.c) < most) poly = std::max(poly, std::fabs(k.b * k.b / (4 * k.c)));
        for (int j = 0; j < n; ++j) next = std::max(next, std::sqrt(at[j]) * std::fabs(k.a + k.b * at[j] + k.c * at[j] * at[j]));
        if (!(next <= kMostSigma) || !(poly <= kMostPoly))
            return fail(AL_EINVAL, "%s: step %d of these coefficients takes singular values to %g, those of b A + c A A to %g (at most %g and %g)", who, i + 1, next, poly,
                        kMostSigma, kMostPoly);
        top = std::max(next, 1e-6);
    }
    return AL_OK;
}

al_status check_sides(int64_t rows, int64_t cols, const char* who) {
    if (rows < 0 || cols < 0) return fail(AL_EINVAL, "%s: negative shape", who);
    if (std::max(rows, cols) > al::kOrthoLong || std::min(rows, cols) > al::kOrthoShort)
        return fail(AL_EUNSUPPORTED, "%s: %lld x %lld is too large", who, (long long)rows, (long long)cols);
    return AL_OK;
}

al::OrthoCoefs coefs(const al_ortho_cfg& k) { return {(float)k.a, (float)k.b, (float)k.c, k.eps, k.steps}; }

bool aligned16(const void* p) { return (at(p) & 15u) == 0; }

// Matrices of a shape that are stepped together.
int64_t batch_of(int64_t rows, int64_t cols) {
    const int64_t n = (rows + 63) / 64 * 64 * ((cols + 63) / 64 * 64);
    return std::max<int64_t>(1, std::min<int64_t>(al::kMuonBatch, (int64_t(1) << 26) / n));
}

al_status check_muon(const al_tensor* ts, int32_t nt, const al_muon_cfg* cfg, const char* who) {
    if (!cfg) return fail(AL_EINVAL, "%s: cfg is NULL", who);
    if (nt < 0) return fail(AL_EINVAL, "%s: nt < 0", who);
    if (nt > 0 && !ts) return fail(AL_EINVAL, "%s: tensors is NULL", who);
    if (!std::isfinite(cfg->lr) || cfg->lr < 0 || !(cfg->beta >= 0 && cfg->beta < 1) || !std::isfinite(cfg->weight_decay) || cfg->weight_decay < 0)
        return fail(AL_EINVAL, "%s: hyperparameters out of range", who);
    if (cfg->nesterov != 0 && cfg->nesterov != 1) return fail(AL_EINVAL, "%s: nesterov %d", who, cfg->nesterov);
    if (cfg->scale < AL_MUON_SCALE_NONE || cfg->scale > AL_MUON_SCALE_RMS) return fail(AL_EINVAL, "%s: scale %d", who, cfg->scale);
    AL_TRY(check_dtype(cfg->grad_dtype, who, "grad_dtype"));
    AL_TRY(check_ortho(cfg->ortho, who));
    if (cfg->m.codec != AL_CODEC_FP32 && cfg->m.codec != AL_CODEC_UF8) return fail(AL_EINVAL, "%s: codec %d not allowed for the momentum", who, cfg->m.codec);
    const bool uf = cfg->m.codec == AL_CODEC_UF8;
    if (uf && cfg->m.block != 256) return fail(AL_EUNSUPPORTED, "%s: UF8 momentum block must be 256 (got %d)", who, cfg->m.block);
    for (int i = 0; i < nt; ++i) {
        const al_tensor& t = ts[i];
        AL_TRY(check_sides(t.rows, t.cols, who));
        if (t.rows == 0 || t.cols == 0) continue;
        if (!t.param || !t.grad || !t.m || (uf && !t.m_meta)) return fail(AL_EINVAL, "tensor %d: param, grad or momentum is NULL", i);
        if (!aligned16(t.param) || !aligned16(t.grad) || !aligned16(t.m) || (uf && !aligned16(t.m_meta)))
            return fail(AL_EALIGN, "tensor %d: param, grad or momentum not 16-byte aligned", i);
        if (t.v || t.v_meta || t.vr || t.vr_meta || t.vc || t.vc_meta || t.cr || t.cr_meta || t.cc || t.cc_meta || (!uf && t.m_meta))
            return fail(AL_EINVAL, "tensor %d: slots besides param, grad and momentum must be NULL for this path", i);
    }
    return AL_OK;
}

// The non-empty tensors by shape, in list order within each.
std::vector<int> by_shape(const al_tensor* ts, int32_t nt) {
    std::vector<int> order;
    for (int i = 0; i < nt; ++i)
        if (ts[i].rows > 0 && ts[i].cols > 0) order.push_back(i);
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) {
        return ts[x].rows != ts[y].rows ? ts[x].rows < ts[y].rows : ts[x].cols < ts[y].cols;
    });
    return order;
}

size_t shape_end(const al_tensor* ts, const std::vector<int>& order, size_t i) {
    size_t j = i;
    while (j < order.size() && ts[order[j]].rows == ts[order[i]].rows && ts[order[j]].cols == ts[order[i]].cols) ++j;
    return j;
}

size_t muon_bytes(const al_tensor* ts, const std::vector<int>& order, int32_t parts) {
    size_t most = 0;
    for (size_t i = 0, j; i < order.size(); i = j) {
        j = shape_end(ts, order, i);
        const al_tensor& t = ts[order[i]];
        // every smaller batch too: it may be cut into more splits
        for (int64_t b = std::min<int64_t>(batch_of(t.rows, t.cols), (int64_t)(j - i)); b > 0; --b)
            most = std::max(most, al::ortho_plan(t.rows, t.cols, parts, (int32_t)b, true).bytes);
    }
    return most;
}

}  // namespace

extern "C" {

al_status al_orthogonalize_workspace_bytes(int64_t rows, int64_t cols, const al_ortho_cfg* cfg, size_t* bytes) {
    const char* const who = "al_orthogonalize_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    if (!cfg) return fail(AL_EINVAL, "%s: cfg is NULL", who);
    AL_TRY(check_ortho(*cfg, who));
    AL_TRY(check_sides(rows, cols, who));
    if (rows > 0 && cols > 0) *bytes = al::ortho_plan(rows, cols, cfg->parts, 1, false).bytes;
    return AL_OK;
}

al_status al_orthogonalize(int32_t dtype, const void* x, int64_t ldx, int64_t rows, int64_t cols, const al_ortho_cfg* cfg, int32_t out_dtype,
                           void* out, int64_t ldout, void* ws, size_t ws_bytes, void* stream) {
    const char* const who = "al_orthogonalize";
    al::api_clear();
    if (!cfg) return fail(AL_EINVAL, "%s: cfg is NULL", who);
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_dtype(out_dtype, who, "out_dtype"));
    AL_TRY(check_ortho(*cfg, who));
    AL_TRY(check_sides(rows, cols, who));
    if (rows == 0 || cols == 0) return AL_OK;
    AL_TRY(check_mat(x, &ldx, rows, cols, dtype, true, who, "x"));
    AL_TRY(check_mat(out, &ldout, rows, cols, out_dtype, true, who, "out"));
    if (x == out && (dtype != out_dtype || ldx != ldout)) return fail(AL_EINVAL, "%s: out may be x with the same type and row pitch only", who);
    const al::OrthoPlan p = al::ortho_plan(rows, cols, cfg->parts, 1, false);
    AL_TRY(check_ws(ws, ws_bytes, p.bytes, who));
    return launched(al::launch_orthogonalize(p, coefs(*cfg), dtype, x, ldx, out_dtype, out, ldout, ws, as_stream(stream)), who);
}

al_status al_muon_workspace_bytes(const al_tensor* tensors, int32_t nt, const al_muon_cfg* cfg, size_t* bytes) {
    const char* const who = "al_muon_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    AL_TRY(check_muon(tensors, nt, cfg, who));
    try {
        *bytes = muon_bytes(tensors, by_shape(tensors, nt), cfg->ortho.parts);
    } catch (const std::bad_alloc&) {
        return fail(AL_EINVAL, "%s: no host memory for a list of %d tensors", who, nt);
    }
    return AL_OK;
}

al_status al_muon_step(const al_tensor* tensors, int32_t nt, const al_muon_cfg* cfg, int64_t step, void* ws, size_t ws_bytes, void* stream) {
    const char* const who = "al_muon_step";
    al::api_clear();
    AL_TRY(check_muon(tensors, nt, cfg, who));
    if (step < 1) return fail(AL_EINVAL, "%s: step must be >= 1", who);
    std::vector<int> order;
    size_t need = 0;
    try {
        order = by_shape(tensors, nt);
        need = muon_bytes(tensors, order, cfg->ortho.parts);
    } catch (const std::bad_alloc&) {
        return fail(AL_EINVAL, "%s: no host memory for a list of %d tensors", who, nt);
    }
    AL_TRY(check_ws(ws, ws_bytes, need, who));
    for (size_t i = 0; i < order.size();) {
        const al_tensor& t = tensors[order[i]];
        const size_t end = std::min(shape_end(tensors, order, i), i + (size_t)batch_of(t.rows, t.cols));
        const al::OrthoPlan p = al::ortho_plan(t.rows, t.cols, cfg->ortho.parts, (int32_t)(end - i), true);
        al::MuonList l = {};
        for (size_t j = i; j < end; ++j) {
            const al_tensor& s = tensors[order[j]];
            l.t[j - i] = {s.param, s.grad, s.m, s.m_meta};
        }
        al::MuonArgs a = {};
        a.beta = cfg->beta;
        a.omb = 1.0 - cfg->beta;
        a.decay = 1.0 - cfg->lr * cfg->weight_decay;
        const double r = (double)t.rows, c = (double)t.cols;
        a.step = cfg->lr * (cfg->scale == AL_MUON_SCALE_NONE ? 1.0 : cfg->scale == AL_MUON_SCALE_SPECTRAL ? std::sqrt(std::max(1.0, r / c)) : 0.2 * std::sqrt(std::max(r, c)));
        a.nesterov = cfg->nesterov;
        a.grad_bf16 = cfg->grad_dtype == AL_DTYPE_BF16;
        a.uf8 = cfg->m.codec == AL_CODEC_UF8;
        AL_TRY(launched(al::launch_muon(p, coefs(cfg->ortho), a, l, ws, as_stream(stream)), who));
        i = end;
    }
    return AL_OK;
}

}  // extern "C"
