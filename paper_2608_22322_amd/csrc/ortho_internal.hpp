// Plan and launchers of the orthogonalised update, shared between the C ABI (ortho_api.cpp, al_api.cpp) and its kernels
// (ortho.hip). Not a public header.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/al.h"

namespace al {

// Most rows and columns, and most on the shorter side (a product's tiles and offsets).
constexpr int64_t kOrthoLong = int64_t(1) << 21, kOrthoShort = int64_t(1) << 16;

struct MmCut {
    int32_t tile, splits;
};
// How a product is cut: a rule on its sizes.
MmCut mm_cut(int64_t m, int64_t n, int64_t turns, int64_t batches, bool sym);
// Bytes of the partial sums of a product cut so.
size_t mm_part_bytes(const MmCut& c, int64_t m, int64_t n, int64_t batches, bool sym);

// Newton-Schulz products over a batch of matrices of one shape. Matrices are held padded with zeros to rp x cp, multiples of
// 64, as one 16-bit part or the sum of two; g1: X X^T (or X^T X), g2: its square, g3: the next X.
struct OrthoPlan {
    int64_t rows, cols;
    int32_t rp, cp, dp, parts, batches;
    bool tall;
    MmCut g1, g2, g3;
    int32_t sums;                                           // partial sums of squares a matrix
    size_t norm_off, sum_off, x0_off, x1_off, a_off, b_off, part_off, bytes;  // regions of the workspace
};
// update: the matrices come as fp32 in the workspace (x0), as al_muon_step forms them.
OrthoPlan ortho_plan(int64_t rows, int64_t cols, int32_t parts, int32_t batches, bool update);

struct OrthoCoefs {
    float a, b, c;
    double eps;
    int32_t steps;
};

// One matrix x (dtype) -> out (out_dtype).
hipError_t launch_orthogonalize(const OrthoPlan& p, const OrthoCoefs& k, int dtype, const void* x, int64_t ldx, int out_dtype, void* out, int64_t ldout,
                                void* ws, hipStream_t st);

// al_muon_step over a batch of tensors of one shape.
constexpr int kMuonBatch = 64;
struct MuonItem {
    float* p;
    const void* g;
    void* m;
    float* meta;
};
struct MuonList {
    MuonItem t[kMuonBatch];
};
struct MuonArgs {
    double beta, omb, decay, step;  // step: lr times the shape's scale
    int32_t nesterov, grad_bf16, uf8;
};
// The momentum pass over `batches` tensors of n elements: u (pitch elements apart) and `parts` partial sums of its squares each, one
// for kMomentum elements.
constexpr int kMomentum = 8192;
hipError_t launch_momentum(const MuonArgs& a, const MuonList& l, int64_t n, int64_t pitch, int32_t parts, int32_t batches, float* u, double* sums,
                           hipStream_t st);
hipError_t launch_muon(const OrthoPlan& p, const OrthoCoefs& k, const MuonArgs& a, const MuonList& l, void* ws, hipStream_t st);

}  // namespace al
