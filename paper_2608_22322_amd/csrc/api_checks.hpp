// Argument checks that the C ABI files share: on the host, before any HIP call.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

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

}  // namespace

#define AL_TRY(x)                              \
    do {                                       \
        const al_status st_ = (x);             \
        if (st_ != AL_OK) return st_;          \
    } while (0)
