// The activation code E8 (save and load) and the gated activation that saves
// and uses it.
//
// All four kernels stream: a lane owns 8 consecutive columns (16 bytes of
// bf16, 8 code bytes), a block of 32, 64 or 128 columns is 4, 8 or 16
// consecutive lanes, and its largest magnitude is a maximum over them in
// registers. Chunks are numbered along the coded rows (pitch / 8 a row), so
// every width fills the wavefronts and a group of lanes never straddles a row.
// Two or four chunks a lane, next to each other or 256 apart, were slower
// (quantize 8192 x 11008: 62 and 63 us against 58; short matrices most of all).
#include <algorithm>

#include "act_device.hpp"

namespace al {

constexpr int kThreads = 256;

struct Grid {
    FastDiv nch;      // chunks per row (pitch / 8)
    uint32_t chunks;  // of this launch, below 2^31
    int64_t row0;     // first row of this launch
};

// A lane's 8 columns. The codec takes its workgroups in XCD order (quantize 8192 x 11008 47.8 -> 46.1 us, dequantize
// 39.2 -> 37.9); the gated activation, with three and five streams, does not (its backward pass 122 -> 141).
struct Place {
    int64_t row;
    int c;
    bool in;  // there is such a chunk (the others stand at the first, and store nothing)
    __device__ __forceinline__ Place(const Grid& g, uint32_t block) {
        const uint32_t q = block * kThreads + threadIdx.x;
        in = q < g.chunks;
        const uint32_t r = quotient(in ? q : 0u, g.nch);
        row = g.row0 + r;
        c = (int)((in ? q : 0u) - r * g.nch.d) * 8;
    }
};

// Matrices pass through once and go past the caches (non-temporal: quantize 58 -> 48 us, dequantize 47 -> 39, the gated
// activation 20.7 -> 17.7 and 143 -> 122); codes are stored for a later reader, who finds small ones in the last-level cache.
template <typename T>
__device__ __forceinline__ void load_mat(Chunk<T>& k, const Mat& m, const Place& at, int cols) {
    load_chunk<T, true>(k, static_cast<const T*>(m.p) + at.row * m.ld, at.c, cols);
}
template <typename T>
__device__ __forceinline__ void store_mat(const Mat& m, const Place& at, int cols, const float (&v)[8]) {
    if (at.in) store_chunk<true>(static_cast<T*>(m.p) + at.row * m.ld, at.c, cols, v);
}

struct Coded {
    u32x2 q;
    uint32_t e;
};
template <bool NT>
__device__ __forceinline__ void load_code(Coded& r, const Code& k, const CodeShape& s, const Place& at) {
    const u32x2* const p = reinterpret_cast<const u32x2*>(k.p + at.row * s.pitch + at.c);
    r.q = NT ? __builtin_nontemporal_load(p) : *p;
    r.e = k.e[at.row * s.nb + (at.c >> (3 + s.lb))];
}

// Codes of a chunk, and by the first lane of a block its exponent. Lanes without a chunk take part in the maximum.
__device__ __forceinline__ void save(const Code& k, const CodeShape& s, const Place& at, const float (&v)[8]) {
    const uint32_t e = e8_exp(group_max(max_bits(v), s.lb));
    if (!at.in) return;
    *reinterpret_cast<u32x2*>(k.p + at.row * s.pitch + at.c) = e8_encode(v, e);
    const int b = at.c >> (3 + s.lb);
    if (at.c == b << (3 + s.lb)) k.e[at.row * s.nb + b] = (uint8_t)e;
}

// 8192 x 11008 bf16: 46 us, 5.9 TB/s; bound by memory.
template <typename T>
__global__ __launch_bounds__(kThreads) void act_quantize_kernel(Mat x, CodeShape s, Code k, Grid g) {
    const Place at(g, xcd_block(blockIdx.x, gridDim.x));
    Chunk<T> raw;
    load_mat<T>(raw, x, at, s.cols);
    float v[8];
    raw.get(v);
    save(k, s, at, v);
}

// 8192 x 11008 to bf16: 38 us, 7.2 TB/s with part of the codes in the last-level cache.
template <typename T>
__global__ __launch_bounds__(kThreads) void act_dequantize_kernel(Code k, CodeShape s, Mat out, Grid g) {
    const Place at(g, xcd_block(blockIdx.x, gridDim.x));
    Coded r;
    load_code<false>(r, k, s, at);
    float v[8];
    e8_decode(r.q, r.e, v);
    store_mat<T>(out, at, s.cols, v);
}

// 1 / (1 + e^-x); 0 where e^-x overflows. For bf16 operands by the hardware's exponential and reciprocal, within (|x| + 5) 2^-24 of
// the value, relative: far inside the outputs' 2^-8. For fp32 to four roundings (2^-22) at any x, which costs nothing beside the
// memory (8192 x 5632 forward 93 us, backward 119; with the hardware's functions 94 and 118).
template <typename T>
__device__ __forceinline__ float sigmoid(float x) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-x));
    return 1.0f / (1.0f + expf(-x));
}

// 2048 x 5632 bf16 with both codes: 17.7 to 18.9 us by device, 5.0 to 5.3 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void swiglu_forward_kernel(Mat gate, Mat up, Mat h, CodeShape s, Code kg, Code ku,
                                                                  Grid g) {
    const Place at(g, blockIdx.x);
    Chunk<T> rg, ru;
    load_mat<T>(rg, gate, at, s.cols);
    load_mat<T>(ru, up, at, s.cols);
    float a[8], b[8], o[8];
    rg.get(a);
    ru.get(b);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = a[j] * sigmoid<T>(a[j]) * b[j];
    store_mat<T>(h, at, s.cols, o);
    if (kg.p) {
        save(kg, s, at, a);
        save(ku, s, at, b);
    }
}

// 8192 x 11008 bf16 with the code of h: 122 to 129 us by device, 6.3 to 6.7 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void swiglu_backward_kernel(Mat dh, Code kg, Code ku, CodeShape s, Mat dgate, Mat dup,
                                                                   Code kh, Grid g) {
    const Place at(g, blockIdx.x);
    Chunk<T> rd;
    Coded rg, ru;
    load_code<true>(rg, kg, s, at);
    load_code<true>(ru, ku, s, at);
    load_mat<T>(rd, dh, at, s.cols);
    float a[8], b[8], d[8], o[8];
    e8_decode(rg.q, rg.e, a);
    e8_decode(ru.q, ru.e, b);
    rd.get(d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float p = sigmoid<T>(a[j]), silu = a[j] * p, du = d[j] * silu;
        o[j] = silu * b[j];
        d[j] = d[j] * b[j] * p * (1.0f + a[j] * (1.0f - p));
        b[j] = du;
    }
    store_mat<T>(dgate, at, s.cols, d);
    store_mat<T>(dup, at, s.cols, b);
    if (kh.p) save(kh, s, at, o);
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
