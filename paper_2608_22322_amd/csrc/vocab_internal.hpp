// Launchers of the token operators (embedding lookup and its gradient, cross entropy of a linear head), shared between their C ABI
// (vocab_api.cpp) and their kernels. Not a public header.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/al.h"
#include "act_internal.hpp"
#include "mm_cut.hpp"

namespace al {

// Token ids or targets, 32 or 64 bits.
struct Ids {
    const void* p;
    int32_t wide;
};

hipError_t launch_embed_forward(int table_dtype, int out_dtype, Mat table, Ids ids, int64_t tokens, int64_t vocab, int32_t cols, float scale, Mat out,
                                hipStream_t st);

// Sorted (id, token) keys in two buffers, where each row's tokens begin among them, and sums of dy over whole pieces of equal ids.
constexpr int kSortRun = 1024, kPiece = 32;
struct EmbedBackward {
    Mat dy;
    Ids ids;
    int64_t tokens, vocab;
    int32_t cols;
    float scale;
    const void* base;
    void* dw;
    uint64_t *key0, *key1;
    uint32_t* begin;
    float* part;
};
struct EmbedPlan {
    size_t key1_off, begin_off, part_off, bytes;
};
EmbedPlan embed_plan(int64_t tokens, int64_t vocab, int64_t cols);
hipError_t launch_embed_backward(int dtype, int grad_dtype, const EmbedBackward& a, hipStream_t st);

// Cross entropy: how a call is cut, by its sizes alone.
struct XentPlan {
    int64_t tokens, hidden, vocab;
    int32_t tp, dp;        // tokens and hidden padded to multiples of 64
    int32_t block, groups; // tokens a pass of the statistics, and the groups of columns that it leaves a row's statistics of
    int32_t piece;         // columns of the vocabulary a pass of the gradients
    int32_t parts, dh_parts, dw_parts;  // of the logits' gradients
    bool pack;             // w is copied into padded rows
    MmCut logits, back, dh, dw;
    size_t h_off, w_off, stat_off, norm_off, coef_off, d_off, dh_off, part_off, bytes;
};
XentPlan xent_plan(int64_t tokens, int64_t hidden, int64_t vocab, int64_t ldw, int dh_dtype, int grad_dtype, bool dh, bool dw);
struct Xent {
    Mat h, w;
    Ids target;
    const float* weight;
    float scale;
    float *loss, *lse;
    Mat dh;
    int32_t dh_bf16, dw_bf16;
    const void* base;
    void* dw;
};
hipError_t launch_xent(const XentPlan& p, const Xent& a, void* ws, hipStream_t st);

}  // namespace al
