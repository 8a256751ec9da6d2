// Launch arguments and launchers of the 8-bit activation operators, shared
// between their C ABI (act_api.cpp) and their kernels. Not a public header.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/al.h"

namespace al {

// The thread's last error (al_last_error): set it, clear it.
al_status api_fail(al_status s, const char* msg);
void api_clear();

// A matrix of the caller's dtype, one row per token.
struct Mat {
    void* p;
    int64_t ld;
};

// An E8 code: rows of `pitch` code bytes and `nb` exponent bytes (p == nullptr: none).
struct Code {
    int8_t* p;
    uint8_t* e;
};

// Geometry of a coded matrix: a block is 2^lb chunks of 8 columns.
struct CodeShape {
    int64_t rows;
    int32_t cols, pitch, nb, lb;
};

inline CodeShape code_shape(int64_t rows, int64_t cols, int32_t block) {
    CodeShape s;
    s.rows = rows;
    s.cols = (int32_t)cols;
    s.nb = (int32_t)((cols + block - 1) / block);
    s.pitch = s.nb * block;
    s.lb = block == 32 ? 2 : block == 64 ? 3 : 4;
    return s;
}

hipError_t launch_act_quantize(int dtype, Mat x, const CodeShape& s, Code c, hipStream_t st);
hipError_t launch_act_dequantize(int dtype, Code c, const CodeShape& s, Mat out, hipStream_t st);
hipError_t launch_swiglu_forward(int dtype, Mat gate, Mat up, Mat h, const CodeShape& s, Code cg, Code cu, hipStream_t st);
hipError_t launch_swiglu_backward(int dtype, Mat dh, Code cg, Code cu, const CodeShape& s, Mat dgate, Mat dup, Code ch,
                                  hipStream_t st);

struct NormForward {
    Mat x, y;
    CodeShape s;  // pitch = cols rounded up to 8 when nothing is saved
    const float *gamma, *beta;
    float *mean, *rstd;
    Code c;
    float eps;
    int64_t row0;  // set by the launcher: a call's first row
};
hipError_t launch_norm_forward(int dtype, bool layer, const NormForward& a, hipStream_t st);

struct NormBackward {
    Mat dy, x, add, dx;
    CodeShape s;
    const float *mean, *rstd, *gamma;
    Code c;
    void *dgamma, *dbeta;
    float* part;  // workspace: [2][parts][cols] partial sums of dgamma, dbeta
    int32_t parts;
    bool grad_bf16;
    int64_t row0;  // set by the launcher: a call's first row
};
// Rows of partial sums that a call writes: a rule on the sizes alone.
int32_t norm_backward_parts(int64_t rows, int64_t cols);
hipError_t launch_norm_backward(int dtype, bool layer, int grad_dtype, const NormBackward& a, hipStream_t st);

struct Wgrad {
    Mat dy;
    CodeShape s;  // rows: tokens, cols: in_features
    int64_t out;  // out_features
    Code c;
    const float *gamma, *beta;
    const void* base;
    void *dw, *dbias;
    float* part;   // workspace: [splits][out][cols] partial products
    float* bsum;   // workspace: out column sums of dy, then [bparts][out] partials (the partials alone if beside)
    int32_t tile, splits, bparts;
    bool beside;    // the sums of dy are taken in the product's launch
    uint32_t sums;  // set by the launcher: how many of that launch's workgroups take them
};
// How a call is cut (tile variant, splits over the tokens), by its sizes alone.
struct WgradPlan {
    int32_t tile, splits, bparts;
    bool beside;
    size_t part_bytes, bsum_bytes;
};
WgradPlan wgrad_plan(int dtype, int64_t tokens, int64_t out, int64_t in);
hipError_t launch_wgrad(int dtype, int grad_dtype, const Wgrad& a, hipStream_t st);

// Sums over the rows of `count` [parts][cols] fp32 arrays, one behind the other, in a fixed order: written as
// grad_dtype to g and as fp32 to f (each where it is not NULL).
struct FoldOut {
    void* g;
    float* f;
};
hipError_t launch_fold(int grad_dtype, const float* part, int32_t parts, int64_t cols, const FoldOut* out, int count, hipStream_t st);

}  // namespace al
