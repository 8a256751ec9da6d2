// The activation code E8 (save and load) and the gated activation that saves
// and uses it.
//
// All four kernels stream: a lane owns chunks of 8 consecutive columns (16
// bytes of bf16, 8 code bytes), a block of 32, 64 or 128 columns is 4, 8 or 16
// consecutive lanes, and its largest magnitude is a maximum over them in
// registers. Chunks are numbered along the coded rows (pitch / 8 a row), so
// every width fills the wavefronts and a group of lanes never straddles a row.
#include <algorithm>

#include "act_device.hpp"

namespace al {

constexpr int kThreads = 256;

struct Grid {
    FastDiv nch;      // chunks per row (pitch / 8)
    uint32_t chunks;  // of this launch, below 2^31
    int64_t row0;     // first row of this launch
};

// The chunk's row and first column.
__device__ __forceinline__ void place(const Grid& g, uint32_t q, int64_t& row, int& c) {
    const uint32_t r = quotient(q, g.nch);
    row = g.row0 + r;
    c = (int)(q - r * g.nch.d) * 8;
}

// Codes of a chunk, and by the first lane of a block its exponent. Lanes without a chunk take part in the maximum.
__device__ __forceinline__ void save(const Code& k, const CodeShape& s, int64_t row, int c, bool in, const float (&v)[8]) {
    const uint32_t e = e8_exp(group_max(max_bits(v), s.lb));
    if (!in) return;
    *reinterpret_cast<u32x2*>(k.p + row * s.pitch + c) = e8_encode(v, e);
    const uint32_t chunk = (uint32_t)c >> 3;
    if ((chunk & ((1u << s.lb) - 1u)) == 0u) k.e[row * s.nb + (chunk >> s.lb)] = (uint8_t)e;
}

__device__ __forceinline__ void load(const Code& k, const CodeShape& s, int64_t row, int c, float (&v)[8]) {
    const u32x2 q = *reinterpret_cast<const u32x2*>(k.p + row * s.pitch + c);
    e8_decode(q, k.e[row * s.nb + (c >> (3 + s.lb))], v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void act_quantize_kernel(Mat x, CodeShape s, Code k, Grid g) {
    const uint32_t q = blockIdx.x * kThreads + threadIdx.x;
    const bool in = q < g.chunks;
    int64_t row;
    int c;
    place(g, in ? q : 0u, row, c);
    Chunk<T> raw;
    load_chunk(raw, static_cast<const T*>(x.p) + row * x.ld, c, s.cols);
    float v[8];
    raw.get(v);
    save(k, s, row, c, in, v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void act_dequantize_kernel(Code k, CodeShape s, Mat out, Grid g) {
    const uint32_t q = blockIdx.x * kThreads + threadIdx.x;
    if (q >= g.chunks) return;
    int64_t row;
    int c;
    place(g, q, row, c);
    if (c >= s.cols) return;
    float v[8];
    load(k, s, row, c, v);
    store_chunk(static_cast<T*>(out.p) + row * out.ld, c, s.cols, v);
}

// 1 / (1 + e^-x); 0 where e^-x overflows. The hardware's exponential and reciprocal: within |x| 2^-24 + 2^-22 of
// the value, relative, far inside a bf16 output's 2^-8.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

template <typename T>
__global__ __launch_bounds__(kThreads) void swiglu_forward_kernel(Mat gate, Mat up, Mat h, CodeShape s, Code kg, Code ku,
                                                                  Grid g) {
    const uint32_t q = blockIdx.x * kThreads + threadIdx.x;
    const bool in = q < g.chunks;
    int64_t row;
    int c;
    place(g, in ? q : 0u, row, c);
    Chunk<T> rg, ru;
    load_chunk(rg, static_cast<const T*>(gate.p) + row * gate.ld, c, s.cols);
    load_chunk(ru, static_cast<const T*>(up.p) + row * up.ld, c, s.cols);
    float a[8], u[8], o[8];
    rg.get(a);
    ru.get(u);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = a[j] * sigmoid(a[j]) * u[j];
    if (in) store_chunk(static_cast<T*>(h.p) + row * h.ld, c, s.cols, o);
    if (kg.p) {
        save(kg, s, row, c, in, a);
        save(ku, s, row, c, in, u);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void swiglu_backward_kernel(Mat dh, Code kg, Code ku, CodeShape s, Mat dgate, Mat dup,
                                                                   Code kh, Grid g) {
    const uint32_t q = blockIdx.x * kThreads + threadIdx.x;
    const bool in = q < g.chunks;
    int64_t row;
    int c;
    place(g, in ? q : 0u, row, c);
    Chunk<T> rd;
    load_chunk(rd, static_cast<const T*>(dh.p) + row * dh.ld, c, s.cols);
    float a[8], u[8], d[8], o[8];
    load(kg, s, row, c, a);
    load(ku, s, row, c, u);
    rd.get(d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float p = sigmoid(a[j]), silu = a[j] * p, du = d[j] * silu;
        o[j] = silu * u[j];
        d[j] = d[j] * u[j] * p * (1.0f + a[j] * (1.0f - p));
        u[j] = du;
    }
    if (in) {
        store_chunk(static_cast<T*>(dgate.p) + row * dgate.ld, c, s.cols, d);
        store_chunk(static_cast<T*>(dup.p) + row * dup.ld, c, s.cols, u);
    }
    if (kh.p) save(kh, s, row, c, in, o);
}

namespace {

// Launches of at most 2^30 chunks each, whole rows.
template <typename F>
hipError_t by_rows(const CodeShape& s, F&& launch) {
    const int64_t nch = s.pitch / 8, most = std::max<int64_t>(1, (int64_t(1) << 30) / nch);
    for (int64_t r = 0; r < s.rows; r += most) {
        Grid g;
        g.nch = fast_div((uint32_t)nch);
        g.chunks = (uint32_t)(std::min(most, s.rows - r) * nch);
        g.row0 = r;
        launch(g, dim3((g.chunks + kThreads - 1) / kThreads));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_act_quantize(int dtype, Mat x, const CodeShape& s, Code c, hipStream_t st) {
    return by_rows(s, [&](const Grid& g, dim3 n) {
        if (dtype == AL_DTYPE_BF16)
            act_quantize_kernel<bf16><<<n, kThreads, 0, st>>>(x, s, c, g);
        else
            act_quantize_kernel<float><<<n, kThreads, 0, st>>>(x, s, c, g);
    });
}

hipError_t launch_act_dequantize(int dtype, Code c, const CodeShape& s, Mat out, hipStream_t st) {
    return by_rows(s, [&](const Grid& g, dim3 n) {
        if (dtype == AL_DTYPE_BF16)
            act_dequantize_kernel<bf16><<<n, kThreads, 0, st>>>(c, s, out, g);
        else
            act_dequantize_kernel<float><<<n, kThreads, 0, st>>>(c, s, out, g);
    });
}

hipError_t launch_swiglu_forward(int dtype, Mat gate, Mat up, Mat h, const CodeShape& s, Code cg, Code cu, hipStream_t st) {
    return by_rows(s, [&](const Grid& g, dim3 n) {
        if (dtype == AL_DTYPE_BF16)
            swiglu_forward_kernel<bf16><<<n, kThreads, 0, st>>>(gate, up, h, s, cg, cu, g);
        else
            swiglu_forward_kernel<float><<<n, kThreads, 0, st>>>(gate, up, h, s, cg, cu, g);
    });
}

hipError_t launch_swiglu_backward(int dtype, Mat dh, Code cg, Code cu, const CodeShape& s, Mat dgate, Mat dup, Code ch,
                                  hipStream_t st) {
    return by_rows(s, [&](const Grid& g, dim3 n) {
        if (dtype == AL_DTYPE_BF16)
            swiglu_backward_kernel<bf16><<<n, kThreads, 0, st>>>(dh, cg, cu, s, dgate, dup, ch, g);
        else
            swiglu_backward_kernel<float><<<n, kThreads, 0, st>>>(dh, cg, cu, s, dgate, dup, ch, g);
    });
}

}  // namespace al
