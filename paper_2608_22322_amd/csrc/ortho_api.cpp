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
al_status check_ortho(const al_ortho_cfg& k, const char* who, double* largest = nullptr) {
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
        if (largest) *largest = std::max(*largest, poly);
        top = std::max(next, 1e-6);
    }
    return AL_OK;
}

al_status check_sides(int64_t rows, int64_t cols, const char* who) {
    if (rows < 0 || cols < 0) return fail(AL_EINVAL, "%s: negative shape", who);
    if (std::max(rows, cols) > al::kOrthoLong || std::min(rows, cols) > al::kOrthoShort || rows * cols > al::kOrthoMost)
        return fail(AL_EUNSUPPORTED, "%s: %lld x %lld is too large", who, (long long)rows, (long long)cols);
    return AL_OK;
}

// Two steps at once hold (a I + B') (a I + B) - a a I as they hold B.
al::OrthoCoefs coefs(const al_ortho_cfg& k) {
    double poly = 0;
    (void)check_ortho(k, "", &poly);
    const double m = std::fabs(k.a) + poly;
    return {(float)k.a, (float)k.b, (float)k.c, k.eps, k.steps, k.parts, m * m + k.a * k.a <= 200.0};
}

bool aligned16(const void* p) { return (at(p) & 15u) == 0; }

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

// The non-empty tensors, longest products first: neighbours share launches.
std::vector<int> by_size(const al_tensor* ts, int32_t nt) {
    std::vector<int> order;
    for (int i = 0; i < nt; ++i)
        if (ts[i].rows > 0 && ts[i].cols > 0) order.push_back(i);
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return std::max(ts[x].rows, ts[x].cols) > std::max(ts[y].rows, ts[y].cols); });
    return order;
}

// One past the last tensor of the group that begins with order[i].
size_t group_end(const al_tensor* ts, const std::vector<int>& order, size_t i, int32_t parts) {
    size_t bytes = 0, j = i;
    for (; j < order.size() && j < i + al::kOrthoGroup; ++j) {
        bytes += al::ortho_item_bytes(ts[order[j]].rows, ts[order[j]].cols, parts, true);
        if (j > i && bytes > al::kOrthoBytes) break;
    }
    return j;
}

// What any group of these tensors, or of some of them, takes: each term grows with the list.
size_t muon_bytes(const al_tensor* ts, int32_t nt, int32_t parts) {
    size_t all = 0, most = 0;
    int64_t sums = 0, turns = 0;
    for (int i = 0; i < nt; ++i) {
        if (ts[i].rows == 0 || ts[i].cols == 0) continue;
        const size_t b = al::ortho_item_bytes(ts[i].rows, ts[i].cols, parts, true);
        all += b;
        most = std::max(most, b);
        sums += al::ortho_sums(ts[i].rows, ts[i].cols);
        turns += al::ortho_turns(ts[i].rows, ts[i].cols, parts);
    }
    if (all == 0) return 0;
    return al::ortho_head_bytes(sums) + al::ortho_part_bytes(turns) + std::min(all, std::max(most, al::kOrthoBytes));
}

size_t ortho_bytes(int64_t rows, int64_t cols, int32_t parts) {
    return al::ortho_head_bytes(al::ortho_sums(rows, cols)) + al::ortho_part_bytes(rows, cols, parts) + al::ortho_item_bytes(rows, cols, parts, false);
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
    if (rows > 0 && cols > 0) *bytes = ortho_bytes(rows, cols, cfg->parts);
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
    AL_TRY(check_ws(ws, ws_bytes, ortho_bytes(rows, cols, cfg->parts), who));
    return launched(al::launch_orthogonalize(rows, cols, coefs(*cfg), dtype, x, ldx, out_dtype, out, ldout, ws, as_stream(stream)), who);
}

al_status al_muon_workspace_bytes(const al_tensor* tensors, int32_t nt, const al_muon_cfg* cfg, size_t* bytes) {
    const char* const who = "al_muon_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    AL_TRY(check_muon(tensors, nt, cfg, who));
    *bytes = muon_bytes(tensors, nt, cfg->ortho.parts);
    return AL_OK;
}

al_status al_muon_step(const al_tensor* tensors, int32_t nt, const al_muon_cfg* cfg, int64_t step, void* ws, size_t ws_bytes, void* stream) {
    const char* const who = "al_muon_step";
    al::api_clear();
    AL_TRY(check_muon(tensors, nt, cfg, who));
    if (step < 1) return fail(AL_EINVAL, "%s: step must be >= 1", who);
    AL_TRY(check_ws(ws, ws_bytes, muon_bytes(tensors, nt, cfg->ortho.parts), who));
    std::vector<int> order;
    try {
        order = by_size(tensors, nt);
    } catch (const std::bad_alloc&) {
        return fail(AL_EINVAL, "%s: no host memory for a list of %d tensors", who, nt);
    }
    al::MuonArgs a = {};
    a.beta = cfg->beta;
    a.omb = 1.0 - cfg->beta;
    a.decay = 1.0 - cfg->lr * cfg->weight_decay;
    a.nesterov = cfg->nesterov;
    a.grad_bf16 = cfg->grad_dtype == AL_DTYPE_BF16;
    a.uf8 = cfg->m.codec == AL_CODEC_UF8;
    for (size_t i = 0; i < order.size();) {
        const size_t end = group_end(tensors, order, i, cfg->ortho.parts);
        al::MuonItem items[al::kOrthoGroup];
        for (size_t j = i; j < end; ++j) {
            const al_tensor& t = tensors[order[j]];
            const double r = (double)t.rows, c = (double)t.cols;
            const double s = cfg->scale == AL_MUON_SCALE_NONE ? 1.0 : cfg->scale == AL_MUON_SCALE_SPECTRAL ? std::sqrt(std::max(1.0, r / c)) : 0.2 * std::sqrt(std::max(r, c));
            items[j - i] = {t.param, t.grad, t.m, t.m_meta, t.rows, t.cols, cfg->lr * s};
        }
        AL_TRY(launched(al::launch_muon(items, (int)(end - i), coefs(cfg->ortho), a, ws, as_stream(stream)), who));
        i = end;
    }
    return AL_OK;
}

}  // extern "C"
