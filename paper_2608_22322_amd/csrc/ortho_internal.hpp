// Plan and launchers of the orthogonalised update, shared between the C ABI (ortho_api.cpp) and its kernels (ortho.hip, muon.hip). Not a public
// header.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/al.h"

namespace al {

// Most rows and columns, most on the shorter side and most elements (a product's tiles and offsets, the grids of the passes over a matrix).
constexpr int64_t kOrthoLong = int64_t(1) << 21, kOrthoShort = int64_t(1) << 16, kOrthoMost = int64_t(1) << 33;

// Matrices whose products share launches: at most kOrthoGroup, and at most kOrthoBytes of workspace where there are several.
constexpr int kOrthoGroup = 32;
constexpr size_t kOrthoBytes = size_t(1) << 30;

// One matrix, held padded with zeros to rp x cp (multiples of 64) as one 16-bit part or the sum of two: X in two places in turn, A = X X^T (or
// X^T X) and B = b A + c A A behind it, and a third place for two steps at once.
struct OrthoItem {
    uint16_t *x[2], *a;
    float* p;     // al_muon_step: the parameters, and lr times the shape's scale
    double step;
    int32_t rows, cols, rp, cp;
};

// Bytes of a matrix in the workspace. update: it comes as fp32 there (in x[0]), as al_muon_step forms it.
size_t ortho_item_bytes(int64_t rows, int64_t cols, int32_t parts, bool update);
// Partial sums of squares of a matrix: one for kSquareUnit elements.
constexpr int64_t kSquareUnit = 8192;
int64_t ortho_sums(int64_t rows, int64_t cols);
// What products that are cut across tiles leave behind: of one matrix, and a bound for a group whose products have `turns` turns of 64 x 64 outputs at
// most, which grows with them.
size_t ortho_part_bytes(int64_t rows, int64_t cols, int32_t parts);
size_t ortho_part_bytes(int64_t turns);
int64_t ortho_turns(int64_t rows, int64_t cols, int32_t parts);
// Bytes in front of the matrices: norms and sums of squares.
size_t ortho_head_bytes(int64_t sums);

struct OrthoCoefs {
    float a, b, c;
    double eps;
    int32_t steps, parts;
    int32_t pairs;  // two steps at once stay within what fp16 holds
};

// One matrix x (dtype) -> out (out_dtype). ws: ortho_head_bytes, ortho_part_bytes and ortho_item_bytes.
hipError_t launch_orthogonalize(int64_t rows, int64_t cols, const OrthoCoefs& k, int dtype, const void* x, int64_t ldx, int out_dtype, void* out, int64_t ldout,
                                void* ws, hipStream_t st);

// A group of al_muon_step.
struct MuonItem {
    float* p;
    const void* g;
    void* m;
    float* meta;
    int64_t rows, cols;
    double step;
};
struct MuonArgs {
    double beta, omb, decay;
    int32_t nesterov, grad_bf16, uf8;
};
hipError_t launch_muon(const MuonItem* items, int count, const OrthoCoefs& k, const MuonArgs& a, void* ws, hipStream_t st);

// The momentum pass over a group: unit u (kSquareUnit elements) of item i is unit begin[i] + u of the launch and leaves its sum of squares there.
struct MomentumItem {
    const void* g;
    void* m;
    float *meta, *u;
    int64_t n;
};
struct MomentumList {
    MomentumItem t[kOrthoGroup];
    uint32_t begin[kOrthoGroup + 1];
    int32_t count;
};
hipError_t launch_momentum(const MuonArgs& a, const MomentumList& l, double* sums, hipStream_t st);

}  // namespace al
