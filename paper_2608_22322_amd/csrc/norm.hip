// Layer and RMS norm over the rows of a matrix, and their backward pass with
// the reduction of the weight gradients.
//
// A group of G lanes (a wavefront, or a workgroup of up to 512) holds one row
// in registers, K chunks of 8 columns per lane, so x is read once and the variance
// is taken about the mean. Rows wider than 16384 columns go through kernels that read
// the row again instead. All of them are bound by memory: 8192 x 4096 bf16 with
// the code of xhat 32 us, 5.3 TB/s; the backward pass from that code, the residual's
// gradient added, 38.7 us, 6.1 TB/s, and 4.7 us for the sums of dgamma; fp32
// rows of 1750 (4096 of them, forward) 13 us.
#include <algorithm>

#include "act_device.hpp"

namespace al {

namespace {

constexpr int kRowMax = 16384;  // widest row held in registers

// Eight floats of a vector of `cols` from c on; `fill` past its end.
__device__ __forceinline__ void load8f(const float* p, int c, int cols, float fill, float (&v)[8]) {
    if (c + 8 <= cols) {
        const u32x4 a = *reinterpret_cast<const u32x4_a4*>(p + c), b = *reinterpret_cast<const u32x4_a4*>(p + c + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = bits_f(a[j]), v[4 + j] = bits_f(b[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? p[c + j] : fill;
    }
}

// Sum over the G lanes of a group, the same in every lane. G > 64: the group is the workgroup; `buf` holds a
// float per wavefront for each of the kernel's sums in turn (double-buffered by the caller).
template <int G>
__device__ __forceinline__ float group_sum(float v, float* buf) {
    v = wave_sum(v);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) v += buf[w];
    }
    return v;
}

// The same sum in the order of a wavefront that holds the row's G / 64 chunks a lane: each lane's chunks first, then the lanes. buf: G floats.
template <int G>
__device__ __forceinline__ float group_sum_by_lane(float v, float* buf) {
    buf[threadIdx.x] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) v += buf[w * 64 + (threadIdx.x & 63)];
    return wave_sum(v);
}

__device__ __forceinline__ float sum8(const float (&v)[8]) {
    return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// Columns of a chunk at c that lie inside the row.
__device__ __forceinline__ int inside(int c, int cols) { return min(8, max(0, cols - c)); }

template <typename T, int G, int K>
__global__ __launch_bounds__(G < 256 ? 256 : G) void norm_forward_kernel(NormForward a, bool layer) {
    constexpr int R = G < 256 ? 256 / G : 1;  // rows per workgroup
    // widths of which many rows take a wavefront each and few a workgroup: a row's bits do not depend on their number
    constexpr bool BY_LANE = sizeof(T) == 2 && G == 256 && K == 1;
    __shared__ float buf[2][BY_LANE ? G : 16];
    const int lane = threadIdx.x % G, cols = a.s.cols;
    const int64_t row = a.row0 + (int64_t)blockIdx.x * R + threadIdx.x / G;
    if (row >= a.s.rows) return;  // a whole group
    const auto row_sum = [&](float v, float* b) {
        if constexpr (BY_LANE) return group_sum_by_lane<G>(v, b);
        else return group_sum<G>(v, b);
    };
    const T* const x = static_cast<const T*>(a.x.p) + row * a.x.ld;
    Chunk<T> raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) load_chunk<T, true>(raw[k], x, (k * G + lane) * 8, cols);
    float v[K][8], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        raw[k].get(v[k]);
        sum += sum8(v[k]);
    }
    float mean = 0.0f;
    if (layer) {
        mean = row_sum(sum, buf[0]) / (float)cols;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int n = inside((k * G + lane) * 8, cols);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = j < n ? v[k][j] - mean : 0.0f;
        }
    }
    float sq = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = v[k][j] * v[k][j];
        sq += sum8(t);
    }
    const float rstd = 1.0f / sqrtf(row_sum(sq, buf[1]) / (float)cols + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* const y = static_cast<T*>(a.y.p) + row * a.y.ld;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + lane) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k][j] *= rstd;
        if (a.c.p) {
            const uint32_t e = e8_exp(group_max(max_bits(v[k]), a.s.lb));
            if (c < a.s.pitch) {
                *reinterpret_cast<u32x2*>(a.c.p + row * a.s.pitch + c) = e8_encode(v[k], e);
                const int b = c >> (3 + a.s.lb);
                if (c == b << (3 + a.s.lb)) a.c.e[row * a.s.nb + b] = (uint8_t)e;
            }
        }
        if (c < cols) {
            float w[8];
            if (a.gamma) {
                load8f(a.gamma, c, cols, 0.0f, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] *= w[j];
            }
            if (a.beta) {
                load8f(a.beta, c, cols, 0.0f, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] += w[j];
            }
            store_chunk<true>(y, c, cols, v[k]);
        }
    }
}

// Rows of any width: one workgroup per row, the row read three times (from the cache after the first). 1024 x 32768 bf16 with the code: 43.5 us,
// 3.9 TB/s.
template <typename T>
__global__ __launch_bounds__(1024) void norm_forward_wide_kernel(NormForward a, bool layer) {
    constexpr int G = 1024;
    __shared__ float buf[2][16];
    const int cols = a.s.cols;
    const int64_t row = a.row0 + blockIdx.x;
    const T* const x = static_cast<const T*>(a.x.p) + row * a.x.ld;
    T* const y = static_cast<T*>(a.y.p) + row * a.y.ld;
    Chunk<T> raw;
    float v[8], mean = 0.0f, sum = 0.0f;
    if (layer) {
        for (int c = threadIdx.x * 8; c < cols; c += G * 8) {
            load_chunk(raw, x, c, cols);
            raw.get(v);
            sum += sum8(v);
        }
        mean = group_sum<G>(sum, buf[0]) / (float)cols;
    }
    sum = 0.0f;
    for (int c = threadIdx.x * 8; c < cols; c += G * 8) {
        load_chunk(raw, x, c, cols);
        raw.get(v);
        const int n = inside(c, cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? (v[j] - mean) * (v[j] - mean) : 0.0f;
        sum += sum8(v);
    }
    const float rstd = 1.0f / sqrtf(group_sum<G>(sum, buf[1]) / (float)cols + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    // the trip count is the same in a whole wavefront, which a block's maximum needs
    for (int c0 = 0; c0 < a.s.pitch; c0 += G * 8) {
        const int c = c0 + threadIdx.x * 8, n = inside(c, cols);
        load_chunk(raw, x, c, cols);
        raw.get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? (v[j] - mean) * rstd : 0.0f;
        if (a.c.p) {
            const uint32_t e = e8_exp(group_max(max_bits(v), a.s.lb));
            if (c < a.s.pitch) {
                *reinterpret_cast<u32x2*>(a.c.p + row * a.s.pitch + c) = e8_encode(v, e);
                const int b = c >> (3 + a.s.lb);
                if (c == b << (3 + a.s.lb)) a.c.e[row * a.s.nb + b] = (uint8_t)e;
            }
        }
        if (c >= cols) continue;
        float w[8];
        if (a.gamma) {
            load8f(a.gamma, c, cols, 0.0f, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= w[j];
        }
        if (a.beta) {
            load8f(a.beta, c, cols, 0.0f, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
        store_chunk(y, c, cols, v);
    }
}

// ------------------------------------------------------------ backward
// What a lane reads of one row's chunk.
template <typename T, bool CODE>
struct RowChunk {
    Chunk<T> dy, x, add;
    u32x2 q;
    uint32_t e;
    __device__ __forceinline__ void load(const NormBackward& a, int64_t row, int c) {
        const int cols = a.s.cols;
        load_chunk<T, true>(dy, static_cast<const T*>(a.dy.p) + row * a.dy.ld, c, cols);
        if constexpr (CODE) {
            q = 0u;
            e = 0u;
            if (c < cols) {
                q = *reinterpret_cast<const u32x2*>(a.c.p + row * a.s.pitch + c);
                e = a.c.e[row * a.s.nb + (c >> (3 + a.s.lb))];
            }
        } else {
            load_chunk<T, true>(x, static_cast<const T*>(a.x.p) + row * a.x.ld, c, cols);
        }
        if (a.add.p) load_chunk<T, true>(add, static_cast<const T*>(a.add.p) + row * a.add.ld, c, cols);
    }
    // xhat; columns past the width give 0
    __device__ __forceinline__ void xhat(float mean, float rstd, int n, float (&v)[8]) const {
        if constexpr (CODE) {
            e8_decode(q, e, v);
        } else {
            x.get(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? (v[j] - mean) * rstd : 0.0f;
        }
    }
};

// Two sums at once over the G lanes of a group; buf: 2 G / 64 floats.
template <int G>
__device__ __forceinline__ void group_sum2(float& u, float& v, float* buf) {
    u = wave_sum(u);
    v = wave_sum(v);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) {
            buf[threadIdx.x >> 6] = u;
            buf[G / 64 + (threadIdx.x >> 6)] = v;
        }
        __syncthreads();
        u = v = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) u += buf[w], v += buf[G / 64 + w];
    }
}

// Rows r0, r0 + gridDim * R, ...: dx of each, and the group's sums over its rows of dy xhat and dy. The next row is
// on its way while one is reduced.
template <typename T, int G, int K, bool CODE, bool LAYER>
__global__ __launch_bounds__(G < 256 ? 256 : G) void norm_backward_kernel(NormBackward a) {
    constexpr int R = G < 256 ? 256 / G : 1;  // rows at a time
    constexpr bool LEAN = K > 2;              // registers for one row: none ahead, gamma read for each
    __shared__ float buf[2][2 * 16];
    __shared__ float fold[R > 1 ? R * G * 8 : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G, cols = a.s.cols;
    const float inv_n = 1.0f / (float)cols;
    float gam[K][8], dg[K][8], db[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + lane) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) gam[k][j] = 1.0f, dg[k][j] = db[k][j] = 0.0f;
        if (!LEAN && a.gamma) load8f(a.gamma, c, cols, 0.0f, gam[k]);
    }
    RowChunk<T, CODE> next[K];
    float next_rstd = 0.0f, next_mean = 0.0f;
    const auto fetch = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < K; ++k) next[k].load(a, row, (k * G + lane) * 8);
        next_rstd = a.rstd[row];
        if (LAYER && !CODE) next_mean = a.mean[row];
    };
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t row = (int64_t)blockIdx.x * R + group;
    if (!LEAN && row < a.s.rows) fetch(row);
    for (int turn = 0; row < a.s.rows; row += step, turn ^= 1) {
        if (LEAN) fetch(row);
        RowChunk<T, CODE> r[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            r[k] = next[k];
            if (LEAN && a.gamma) load8f(a.gamma, (k * G + lane) * 8, cols, 0.0f, gam[k]);
        }
        const float rstd = next_rstd, mean = next_mean;
        if (!LEAN && row + step < a.s.rows) fetch(row + step);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float xh[8], dy[8], t[8], u[8];
            r[k].xhat(mean, rstd, inside((k * G + lane) * 8, cols), xh);
            r[k].dy.get(dy);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dg[k][j] += dy[j] * xh[j];
                if (LAYER) db[k][j] += dy[j];
                t[j] = dy[j] * gam[k][j];
                u[j] = t[j] * xh[j];
            }
            s1 += sum8(t);
            s2 += sum8(u);
        }
        if (LAYER)
            group_sum2<G>(s1, s2, buf[turn]);
        else
            s2 = group_sum<G>(s2, buf[turn]);
        s1 *= inv_n;
        s2 *= inv_n;
        T* const dx = static_cast<T*>(a.dx.p) + row * a.dx.ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * 8;
            float xh[8], v[8];
            r[k].xhat(mean, rstd, inside(c, cols), xh);
            r[k].dy.get(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = v[j] * gam[k][j] - xh[j] * s2;
                if (LAYER) v[j] -= s1;
                v[j] *= rstd;
            }
            if (a.add.p) {
                float w[8];
                r[k].add.get(w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += w[j];
            }
            if (c < cols) store_chunk<true>(dx, c, cols, v);
        }
    }
    if (!a.part) return;
    // the workgroup's sums: its R groups in order, then one row of partials each for dgamma and dbeta (or, of a single
    // workgroup, the gradients themselves)
    for (int which = 0; which < (LAYER ? 2 : 1); ++which) {
        float* const out = a.part + ((int64_t)which * a.parts + blockIdx.x) * cols;
        void* const grad = which ? a.dbeta : a.dgamma;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * 8;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = which ? db[k][j] : dg[k][j];
            if constexpr (R > 1) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) fold[(group * 8 + j) * G + lane] = v[j];
                __syncthreads();
                if (group == 0) {
#pragma unroll
                    for (int g = 1; g < R; ++g)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += fold[(g * 8 + j) * G + lane];
                }
            }
            if (group != 0 || c >= cols) continue;
            if (a.parts > 1)
                store_chunk(out, c, cols, v);
            else if (grad && a.grad_bf16)
                store_chunk(static_cast<bf16*>(grad), c, cols, v);
            else if (grad)
                store_chunk(static_cast<float*>(grad), c, cols, v);
        }
    }
}

// Rows of any width: dx alone, one workgroup per row, its row read twice. 1024 x 32768 bf16 from the code: 51 us, and 19 for the weight
// gradients below and 5 for their sums.
template <typename T, bool CODE, bool LAYER>
__global__ __launch_bounds__(1024) void norm_backward_wide_kernel(NormBackward a) {
    constexpr int G = 1024;
    __shared__ float buf[2][16];
    const int cols = a.s.cols;
    const int64_t row = a.row0 + blockIdx.x;
    const float rstd = a.rstd[row], mean = LAYER && !CODE ? a.mean[row] : 0.0f, inv_n = 1.0f / (float)cols;
    T* const dx = static_cast<T*>(a.dx.p) + row * a.dx.ld;
    RowChunk<T, CODE> r;
    float s1 = 0.0f, s2 = 0.0f, xh[8], dy[8], gam[8];
    for (int c = threadIdx.x * 8; c < cols; c += G * 8) {
        r.load(a, row, c);
        r.xhat(mean, rstd, inside(c, cols), xh);
        r.dy.get(dy);
        float t[8], u[8];
        if (a.gamma) load8f(a.gamma, c, cols, 0.0f, gam);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t[j] = a.gamma ? dy[j] * gam[j] : dy[j];
            u[j] = t[j] * xh[j];
        }
        s1 += sum8(t);
        s2 += sum8(u);
    }
    s1 = LAYER ? group_sum<G>(s1, buf[0]) * inv_n : 0.0f;
    s2 = group_sum<G>(s2, buf[1]) * inv_n;
    for (int c = threadIdx.x * 8; c < cols; c += G * 8) {
        r.load(a, row, c);
        r.xhat(mean, rstd, inside(c, cols), xh);
        r.dy.get(dy);
        if (a.gamma) load8f(a.gamma, c, cols, 0.0f, gam);
        float w[8], v[8];
        if (a.add.p) r.add.get(w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = ((a.gamma ? dy[j] * gam[j] : dy[j]) - xh[j] * s2 - s1) * rstd;
            if (a.add.p) v[j] += w[j];
        }
        store_chunk(dx, c, cols, v);
    }
}

// The weight gradients of wide rows: a lane holds 8 columns, a workgroup (blockIdx.y) every parts-th row.
template <typename T, bool CODE, bool LAYER>
__global__ __launch_bounds__(64) void norm_weights_wide_kernel(NormBackward a) {
    const int cols = a.s.cols, c = (blockIdx.x * 64 + threadIdx.x) * 8;
    if (c >= cols) return;
    a.add.p = nullptr;
    float dg[8] = {}, db[8] = {};
    for (int64_t row = blockIdx.y; row < a.s.rows; row += a.parts) {
        RowChunk<T, CODE> r;
        r.load(a, row, c);
        float xh[8], dy[8];
        r.xhat(LAYER && !CODE ? a.mean[row] : 0.0f, a.rstd[row], inside(c, cols), xh);
        r.dy.get(dy);
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[j] += dy[j] * xh[j], db[j] += dy[j];
    }
    store_chunk(a.part + (int64_t)blockIdx.y * cols, c, cols, dg);
    if (LAYER) store_chunk(a.part + ((int64_t)a.parts + blockIdx.y) * cols, c, cols, db);
}

// Column sums of partial sums, from column c0 on: 64 columns a workgroup, wavefront w of 16 takes rows w, w + 16, ..., 8 of them in
// flight.
template <typename O>
__global__ __launch_bounds__(1024) void fold_kernel(const float* part, int32_t parts, int64_t cols, int64_t c0, FoldOut o0, FoldOut o1) {
    __shared__ float buf[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = c0 + (int64_t)blockIdx.x * 64 + lane;
    const FoldOut o = blockIdx.y ? o1 : o0;
    const float* const p0 = part + (int64_t)blockIdx.y * parts * cols + c;
    float s = 0.0f;
    if (c < cols) {
        int p = w;
        float t[8] = {};
        for (; p + 112 < parts; p += 128)
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] += p0[(int64_t)(p + 16 * i) * cols];
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (p + 16 * i < parts) t[i] += p0[(int64_t)(p + 16 * i) * cols];
        s = sum8(t);
    }
    buf[w][lane] = s;
    __syncthreads();
    if (w > 0 || c >= cols) return;
    float a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = buf[i][lane] + buf[i + 8][lane];
    s = sum8(a);
    if (o.g) put(static_cast<O*>(o.g) + c, s);
    if (o.f) o.f[c] = s;
}

// Lanes and chunks per lane that hold a row of `chunks` chunks.
struct Shape {
    int g, k;
};
Shape row_shape(int64_t chunks) {
    if (chunks <= 64) return {64, 1};
    if (chunks <= 128) return {64, 2};
    if (chunks <= 256) return {256, 1};
    if (chunks <= 512) return {256, 2};
    return {512, chunks <= 1024 ? 2 : chunks <= 1536 ? 3 : 4};
}

constexpr int64_t kSlab = 1 << 21;  // rows of one launch (a grid holds fewer than 2^32 threads)

template <typename T>
hipError_t forward_slab(bool layer, const NormForward& a, int64_t rows, hipStream_t st) {
    if (a.s.pitch > kRowMax) {
        norm_forward_wide_kernel<T><<<dim3((uint32_t)rows), 1024, 0, st>>>(a, layer);
        return hipGetLastError();
    }
    Shape s = row_shape(a.s.pitch / 8);
    // bf16 rows of 1025 to 2048 columns: a wavefront each needs no barrier, but walks four chunks a lane one after another, which many rows
    // hide and few do not (RMS with the code, a wavefront a row and a workgroup a row, us in a graph: 8192 x 1100 11.7 and 16.6, 4096 x 2048 7.9
    // and 10.2, 2048 x 1032 5.1 and 5.5, 2048 x 1100 6.1 and 5.8, 2048 x 2048 5.8 and 5.9, 1024 x 1536 4.7 and 3.9, 1 x 2048 3.8 and 2.5).
    // With 8 chunks a lane (8192 x 4096) or fp32 there is nothing in it, or less.
    if (sizeof(T) == 2 && s.g == 256 && s.k == 1 && a.s.rows >= 2048) s = {64, 4};
    const dim3 n((uint32_t)(s.g == 64 ? (rows + 3) / 4 : rows));
    if (s.g == 64 && s.k == 1)
        norm_forward_kernel<T, 64, 1><<<n, 256, 0, st>>>(a, layer);
    else if (s.g == 64 && s.k == 2)
        norm_forward_kernel<T, 64, 2><<<n, 256, 0, st>>>(a, layer);
    else if (s.g == 256 && s.k == 1)
        norm_forward_kernel<T, 256, 1><<<n, 256, 0, st>>>(a, layer);
    else if (s.g == 256 && s.k == 2)
        norm_forward_kernel<T, 256, 2><<<n, 256, 0, st>>>(a, layer);
    else if (s.g == 512 && s.k == 2)
        norm_forward_kernel<T, 512, 2><<<n, 512, 0, st>>>(a, layer);
    else if (s.g == 512 && s.k == 3)
        norm_forward_kernel<T, 512, 3><<<n, 512, 0, st>>>(a, layer);
    else if (s.g == 512 && s.k == 4)
        norm_forward_kernel<T, 512, 4><<<n, 512, 0, st>>>(a, layer);
    if constexpr (sizeof(T) == 2)
        if (s.g == 64 && s.k == 4) norm_forward_kernel<T, 64, 4><<<n, 256, 0, st>>>(a, layer);
    return hipGetLastError();
}

template <typename T>
hipError_t forward(bool layer, NormForward a, hipStream_t st) {
    hipError_t e = hipSuccess;
    for (a.row0 = 0; a.row0 < a.s.rows && e == hipSuccess; a.row0 += kSlab)
        e = forward_slab<T>(layer, a, std::min(kSlab, a.s.rows - a.row0), st);
    return e;
}

template <typename T, bool CODE, bool LAYER>
hipError_t backward(NormBackward a, hipStream_t st) {
    if (a.s.cols > kRowMax) {
        for (a.row0 = 0; a.row0 < a.s.rows; a.row0 += kSlab)
            norm_backward_wide_kernel<T, CODE, LAYER><<<dim3((uint32_t)std::min(kSlab, a.s.rows - a.row0)), 1024, 0, st>>>(a);
        if (a.part)
            norm_weights_wide_kernel<T, CODE, LAYER><<<dim3((uint32_t)((a.s.cols + 511) / 512), (uint32_t)a.parts), 64, 0, st>>>(a);
        return hipGetLastError();
    }
    const Shape s = row_shape((a.s.cols + 7) / 8);
    const dim3 n((uint32_t)a.parts);
    if (s.g == 64 && s.k == 1)
        norm_backward_kernel<T, 64, 1, CODE, LAYER><<<n, 256, 0, st>>>(a);
    else if (s.g == 64 && s.k == 2)
        norm_backward_kernel<T, 64, 2, CODE, LAYER><<<n, 256, 0, st>>>(a);
    else if (s.g == 256 && s.k == 1)
        norm_backward_kernel<T, 256, 1, CODE, LAYER><<<n, 256, 0, st>>>(a);
    else if (s.g == 256 && s.k == 2)
        norm_backward_kernel<T, 256, 2, CODE, LAYER><<<n, 256, 0, st>>>(a);
    else if (s.g == 512 && s.k == 2)
        norm_backward_kernel<T, 512, 2, CODE, LAYER><<<n, 512, 0, st>>>(a);
    else if (s.g == 512 && s.k == 3)
        norm_backward_kernel<T, 512, 3, CODE, LAYER><<<n, 512, 0, st>>>(a);
    else if (s.g == 512 && s.k == 4)
        norm_backward_kernel<T, 512, 4, CODE, LAYER><<<n, 512, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(bool layer, const NormBackward& a, hipStream_t st) {
    if (a.c.p) return layer ? backward<T, true, true>(a, st) : backward<T, true, false>(a, st);
    return layer ? backward<T, false, true>(a, st) : backward<T, false, false>(a, st);
}

}  // namespace

hipError_t launch_fold(int grad_dtype, const float* part, int32_t parts, int64_t cols, const FoldOut* out, int count, hipStream_t st) {
    constexpr int64_t kMost = int64_t(1) << 27;  // columns of one launch (16 threads each; a grid holds fewer than 2^32)
    const FoldOut &a = out[0], &b = out[count - 1];
    for (int64_t c0 = 0; c0 < cols; c0 += kMost) {
        const dim3 n((uint32_t)((std::min(kMost, cols - c0) + 63) / 64), (uint32_t)count);
        if (grad_dtype == AL_DTYPE_BF16)
            fold_kernel<bf16><<<n, 1024, 0, st>>>(part, parts, cols, c0, a, b);
        else
            fold_kernel<float><<<n, 1024, 0, st>>>(part, parts, cols, c0, a, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_norm_forward(int dtype, bool layer, const NormForward& a, hipStream_t st) {
    return dtype == AL_DTYPE_BF16 ? forward<bf16>(layer, a, st) : forward<float>(layer, a, st);
}

// Workgroups of the backward pass, each of which leaves a row of partial weight gradients: few enough that these stay a small part
// of what moves, enough to keep rows in flight (8192 x 4096 bf16: 384 workgroups 42 us, 512 39, 768 40, 1024 44; rows held by
// a wavefront, 16384 x 500: 512 37, 1024 29, 2048 36). Up to 8 turns go to one workgroup, which needs no second
// launch (8 rows of 4096: 11.3 and 12.1 us a call).
int32_t norm_backward_parts(int64_t rows, int64_t cols) {
    if (cols > kRowMax) return (int32_t)std::min<int64_t>(rows, 64);
    const bool waves = row_shape((cols + 7) / 8).g == 64;
    const int64_t turns = waves ? (rows + 3) / 4 : rows, most = waves ? 1024 : 512;
    return (int32_t)(turns <= 8 ? std::min<int64_t>(turns, 1) : std::min(turns, most));
}

hipError_t launch_norm_backward(int dtype, bool layer, int grad_dtype, const NormBackward& a, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (a.s.rows > 0) e = dtype == AL_DTYPE_BF16 ? backward<bf16>(layer, a, st) : backward<float>(layer, a, st);
    // (without rows there is no workspace either, and the sums are zeros)
    if (e == hipSuccess && (a.dgamma || a.dbeta) && (a.parts != 1 || a.s.cols > kRowMax)) {
        const FoldOut out[2] = {{a.dgamma, nullptr}, {a.dbeta, nullptr}};
        e = launch_fold(grad_dtype, a.part, a.parts, a.s.cols, out, layer ? 2 : 1, st);
    }
    return e;
}

}  // namespace al
