// C ABI of the token operators: argument checks on the host before any HIP call, workspace layout, launches on the caller's stream. See include/al.h for
// the contract of each entry point.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "api_checks.hpp"
#include "vocab_internal.hpp"

namespace {

// Most entries of a table that is looked up, of one with a gradient (a grid of rows), most tokens or entries and most features of a head (offsets inside a
// tile's operands are 32 bits).
constexpr int64_t kMostIds = (int64_t(1) << 31) - 1, kMostRowsOfGrad = int64_t(1) << 26, kMostSide = int64_t(1) << 24, kMostHidden = int64_t(1) << 22;

al_status check_index(int32_t d, const char* who) {
    if (d != AL_INDEX_I32 && d != AL_INDEX_I64) return fail(AL_EINVAL, "%s: index_dtype %d", who, d);
    return AL_OK;
}

al_status check_ids(const void* p, int32_t index, const char* who, const char* name) {
    if (!p) return fail(AL_EINVAL, "%s: %s is NULL", who, name);
    if (at(p) & (index == AL_INDEX_I64 ? 7u : 3u)) return fail(AL_EALIGN, "%s: %s is not aligned to its type", who, name);
    return AL_OK;
}

al_status check_sizes(int64_t tokens, int64_t vocab, int64_t cols, const char* who) {
    if (vocab < 0) return fail(AL_EINVAL, "%s: negative shape", who);
    if (vocab > kMostIds) return fail(AL_EUNSUPPORTED, "%s: a vocabulary of %lld is too large", who, (long long)vocab);
    return check_shape(tokens, cols, who);
}

// A weight gradient and what it is added to.
al_status check_packed(const void* dw, const void* base, int64_t rows, int64_t cols, const char* who) {
    if (!dw) return fail(AL_EINVAL, "%s: dw is NULL", who);
    if ((at(dw) | at(base)) & 15u) return fail(AL_EALIGN, "%s: dw or base not 16-byte aligned", who);
    if (cols > 0 && rows > (int64_t(1) << 48) / cols) return fail(AL_EUNSUPPORTED, "%s: dw spans too much memory", who);
    return AL_OK;
}

// The grids of the table's gradient: rows by 1024 columns, and a workgroup for every 32 tokens of 1024 columns, fewer than 2^23 of these.
al_status check_grad(int64_t tokens, int64_t vocab, int64_t cols, const char* who) {
    const int64_t slabs = (cols + 1023) / 1024;
    if (vocab > kMostRowsOfGrad || slabs > 65535 || (slabs > 0 && tokens / 32 >= (int64_t(1) << 23) / slabs))
        return fail(AL_EUNSUPPORTED, "%s: %lld tokens, a table of %lld x %lld are too large", who, (long long)tokens, (long long)vocab, (long long)cols);
    return AL_OK;
}

al_status check_scale(double scale, const char* who) {
    if (!std::isfinite((float)scale)) return fail(AL_EINVAL, "%s: scale must be finite in fp32", who);
    return AL_OK;
}

al_status check_xent(int64_t tokens, int64_t hidden, int64_t vocab, const char* who) {
    if (tokens < 0 || hidden < 0 || vocab < 0) return fail(AL_EINVAL, "%s: negative shape", who);
    constexpr int64_t most = int64_t(1) << 34;
    if (tokens > kMostSide || hidden > kMostHidden || vocab > kMostSide || tokens * vocab > (int64_t(1) << 38) || tokens * hidden > most || vocab * hidden > most)
        return fail(AL_EUNSUPPORTED, "%s: %lld tokens, %lld features, a vocabulary of %lld are too large", who, (long long)tokens, (long long)hidden, (long long)vocab);
    if (hidden == 0 || vocab == 0) return fail(AL_EINVAL, "%s: no logits without features and a vocabulary", who);
    return AL_OK;
}

al::Mat mat(const void* p, int64_t ld) { return {const_cast<void*>(p), ld}; }

}  // namespace

extern "C" {

al_status al_embed_forward(int32_t table_dtype, const void* table, int64_t ldtable, int64_t vocab, int64_t cols, int32_t index_dtype,
                           const void* ids, int64_t tokens, double scale, int32_t out_dtype, void* out, int64_t ldout, void* stream) {
    const char* const who = "al_embed_forward";
    al::api_clear();
    AL_TRY(check_dtype(table_dtype, who, "table_dtype"));
    AL_TRY(check_dtype(out_dtype, who, "out_dtype"));
    AL_TRY(check_index(index_dtype, who));
    AL_TRY(check_sizes(tokens, vocab, cols, who));
    AL_TRY(check_scale(scale, who));
    if (tokens == 0 || cols == 0) return AL_OK;
    AL_TRY(check_ids(ids, index_dtype, who, "ids"));
    AL_TRY(check_mat(table, &ldtable, vocab, cols, table_dtype, vocab > 0, who, "table"));
    AL_TRY(check_mat(out, &ldout, tokens, cols, out_dtype, true, who, "out"));
    return launched(al::launch_embed_forward(table_dtype, out_dtype, mat(table, ldtable), al::Ids{ids, index_dtype == AL_INDEX_I64}, tokens, vocab, (int32_t)cols,
                                             (float)scale, mat(out, ldout), as_stream(stream)), who);
}

al_status al_embed_backward_workspace_bytes(int64_t tokens, int64_t vocab, int64_t cols, size_t* bytes) {
    const char* const who = "al_embed_backward_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    AL_TRY(check_sizes(tokens, vocab, cols, who));
    AL_TRY(check_grad(tokens, vocab, cols, who));
    *bytes = al::embed_plan(tokens, vocab, cols).bytes;
    return AL_OK;
}

al_status al_embed_backward(int32_t dtype, const void* dy, int64_t lddy, int32_t index_dtype, const void* ids, int64_t tokens, int64_t vocab,
                            int64_t cols, double scale, int32_t grad_dtype, const void* base, void* dw, void* ws, size_t ws_bytes, void* stream) {
    const char* const who = "al_embed_backward";
    al::api_clear();
    AL_TRY(check_dtype(dtype, who, "dtype"));
    AL_TRY(check_dtype(grad_dtype, who, "grad_dtype"));
    AL_TRY(check_index(index_dtype, who));
    AL_TRY(check_sizes(tokens, vocab, cols, who));
    AL_TRY(check_grad(tokens, vocab, cols, who));
    AL_TRY(check_scale(scale, who));
    if (vocab == 0 || cols == 0) return AL_OK;
    AL_TRY(check_packed(dw, base, vocab, cols, who));
    if (tokens > 0) {
        AL_TRY(check_ids(ids, index_dtype, who, "ids"));
        AL_TRY(check_mat(dy, &lddy, tokens, cols, dtype, true, who, "dy"));
    }
    const al::EmbedPlan p = al::embed_plan(tokens, vocab, cols);
    AL_TRY(check_ws(ws, ws_bytes, p.bytes, who));
    char* const w = static_cast<char*>(ws);
    al::EmbedBackward a;
    std::memset(&a, 0, sizeof(a));
    a.dy = mat(dy, lddy);
    a.ids = {ids, index_dtype == AL_INDEX_I64};
    a.tokens = tokens;
    a.vocab = vocab;
    a.cols = (int32_t)cols;
    a.scale = (float)scale;
    a.base = base;
    a.dw = dw;
    a.key0 = reinterpret_cast<uint64_t*>(w);
    a.key1 = reinterpret_cast<uint64_t*>(w + p.key1_off);
    a.begin = reinterpret_cast<uint32_t*>(w + p.begin_off);
    a.part = reinterpret_cast<float*>(w + p.part_off);
    return launched(al::launch_embed_backward(dtype, grad_dtype, a, as_stream(stream)), who);
}

al_status al_linear_xent_workspace_bytes(int64_t tokens, int64_t hidden, int64_t vocab, int64_t ldw, int32_t want_dh, int32_t dh_dtype,
                                         int32_t want_dw, int32_t grad_dtype, size_t* bytes) {
    const char* const who = "al_linear_xent_workspace_bytes";
    al::api_clear();
    if (!bytes) return fail(AL_EINVAL, "%s: bytes is NULL", who);
    *bytes = 0;
    AL_TRY(check_xent(tokens, hidden, vocab, who));
    AL_TRY(check_dtype(dh_dtype, who, "dh_dtype"));
    AL_TRY(check_dtype(grad_dtype, who, "grad_dtype"));
    if (vocab <= 1) ldw = hidden;
    if (ldw < hidden) return fail(AL_EINVAL, "%s: w has row pitch %lld < %lld columns", who, (long long)ldw, (long long)hidden);
    if (tokens > 0) *bytes = al::xent_plan(tokens, hidden, vocab, ldw, dh_dtype, grad_dtype, want_dh != 0, want_dw != 0).bytes;
    return AL_OK;
}

al_status al_linear_xent(const void* h, int64_t ldh, const void* w, int64_t ldw, int64_t tokens, int64_t hidden, int64_t vocab,
                         int32_t index_dtype, const void* target, const float* weight, double scale, float* loss, float* lse, int32_t dh_dtype, void* dh,
                         int64_t lddh, int32_t grad_dtype, const void* base, void* dw, void* ws, size_t ws_bytes, void* stream) {
    const char* const who = "al_linear_xent";
    al::api_clear();
    AL_TRY(check_xent(tokens, hidden, vocab, who));
    AL_TRY(check_dtype(dh_dtype, who, "dh_dtype"));
    AL_TRY(check_dtype(grad_dtype, who, "grad_dtype"));
    AL_TRY(check_index(index_dtype, who));
    AL_TRY(check_scale(scale, who));
    if (dw)
        AL_TRY(check_packed(dw, base, vocab, hidden, who));
    else if (base)
        return fail(AL_EINVAL, "%s: base goes with dw", who);
    if (tokens == 0) {  // no token: dw is the base
        if (!dw || dw == base) return AL_OK;
        al::EmbedBackward a;
        std::memset(&a, 0, sizeof(a));
        a.vocab = vocab;
        a.cols = (int32_t)hidden;
        a.base = base;
        a.dw = dw;
        return launched(al::launch_embed_backward(AL_DTYPE_BF16, grad_dtype, a, as_stream(stream)), who);
    }
    AL_TRY(check_mat(h, &ldh, tokens, hidden, AL_DTYPE_BF16, true, who, "h"));
    AL_TRY(check_mat(w, &ldw, vocab, hidden, AL_DTYPE_BF16, true, who, "w"));
    if (at(w) & 15u) return fail(AL_EALIGN, "%s: w not 16-byte aligned", who);
    AL_TRY(check_ids(target, index_dtype, who, "target"));
    AL_TRY(check_vec(weight, AL_DTYPE_F32, who, "weight"));
    AL_TRY(check_vec(loss, AL_DTYPE_F32, who, "loss"));
    AL_TRY(check_vec(lse, AL_DTYPE_F32, who, "lse"));
    AL_TRY(check_mat(dh, &lddh, tokens, hidden, dh_dtype, false, who, "dh"));
    if ((dh && (dh == h || dh == w)) || (dw && (dw == h || dw == w))) return fail(AL_EINVAL, "%s: gradients must not be h or w", who);
    const al::XentPlan p = al::xent_plan(tokens, hidden, vocab, ldw, dh_dtype, grad_dtype, dh != nullptr, dw != nullptr);
    AL_TRY(check_ws(ws, ws_bytes, p.bytes, who));
    al::Xent a;
    std::memset(&a, 0, sizeof(a));
    a.h = mat(h, ldh);
    a.w = mat(w, ldw);
    a.target = {target, index_dtype == AL_INDEX_I64};
    a.weight = weight;
    a.scale = (float)scale;
    a.loss = loss;
    a.lse = lse;
    a.dh = mat(dh, lddh);
    a.dh_bf16 = dh_dtype == AL_DTYPE_BF16;
    a.dw_bf16 = grad_dtype == AL_DTYPE_BF16;
    a.base = base;
    a.dw = dw;
    return launched(al::launch_xent(p, a, ws, as_stream(stream)), who);
}

}  // extern "C"
