// Device helpers of the 8-bit activation operators: chunks of 8 columns, the
// E8 code, sums and maxima over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "act_internal.hpp"

namespace al {

struct bf16 {
    uint16_t b;
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Loads and stores of a chunk at the element's own alignment (the hardware takes unaligned 16-byte
// accesses; rows of odd pitch need them).
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float bits_f(uint32_t u) { return __uint_as_float(u); }
__device__ __forceinline__ uint32_t f_bits(float f) { return __float_as_uint(f); }

__device__ __forceinline__ float to_f(bf16 v) { return bits_f((uint32_t)v.b << 16); }
__device__ __forceinline__ float to_f(float v) { return v; }

// Round to nearest even; NaN stays NaN.
__device__ __forceinline__ uint16_t round_bf16(float f) {
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ void put(bf16* p, float v) { p->b = round_bf16(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// A raw chunk of 8 elements, so that loads can be issued before they are used.
template <typename T>
struct Chunk;
template <>
struct Chunk<bf16> {
    u32x4 q;
    __device__ __forceinline__ void load(const bf16* p) { q = *reinterpret_cast<const u32x4_a2*>(p); }
    __device__ __forceinline__ void load_nt(const bf16* p) { q = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p)); }
    // the first n of 8 elements, the others 0
    __device__ __forceinline__ void load(const bf16* p, int n) {
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = j < n ? p[j].b : 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = h[2 * j] | (h[2 * j + 1] << 16);
    }
    __device__ __forceinline__ void zero() { q = 0u; }
    // drop the first n of 8 elements, the rest moves down and zeros follow
    __device__ __forceinline__ void drop(int n) {
        if (n & 4) q = u32x4{q[2], q[3], 0u, 0u};
        if (n & 2) q = u32x4{q[1], q[2], q[3], 0u};
        if (n & 1) q = u32x4{(q[0] >> 16) | (q[1] << 16), (q[1] >> 16) | (q[2] << 16), (q[2] >> 16) | (q[3] << 16), q[3] >> 16};
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bits_f(q[j] << 16);
            v[2 * j + 1] = bits_f(q[j] & 0xffff0000u);
        }
    }
};
template <>
struct Chunk<float> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const u32x4_a4*>(p);
        b = *reinterpret_cast<const u32x4_a4*>(p + 4);
    }
    // two loads share each line here, and the second finds it only if the first let it in
    __device__ __forceinline__ void load_nt(const float* p) { load(p); }
    __device__ __forceinline__ void load(const float* p, int n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = j < n ? f_bits(p[j]) : 0u;
            b[j] = j + 4 < n ? f_bits(p[j + 4]) : 0u;
        }
    }
    __device__ __forceinline__ void zero() { a = 0u, b = 0u; }
    __device__ __forceinline__ void drop(int n) {
        if (n & 4) a = b, b = 0u;
        if (n & 2) a = u32x4{a[2], a[3], b[0], b[1]}, b = u32x4{b[2], b[3], 0u, 0u};
        if (n & 1) a = u32x4{a[1], a[2], a[3], b[0]}, b = u32x4{b[1], b[2], b[3], 0u};
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = bits_f(a[j]);
            v[j + 4] = bits_f(b[j]);
        }
    }
};

// NT: past the caches, for what passes through once (bf16; fp32 keeps ordinary accesses: saving and loading 8192 x 5632
// 88 us, past the caches 108).
// Load the chunk at columns c .. c + 7 of a row of `cols`; columns past it read as 0. (The chunk that the row ends in is
// taken from the row's last 8 columns: one load instead of up to seven.)
template <typename T, bool NT = false>
__device__ __forceinline__ void load_chunk(Chunk<T>& k, const T* row, int c, int cols) {
    if (c + 8 <= cols) {
        if (NT)
            k.load_nt(row + c);
        else
            k.load(row + c);
    } else if (c >= cols) {
        k.zero();
    } else if (cols >= 8) {
        k.load(row + cols - 8);
        k.drop(c + 8 - cols);
    } else {
        k.load(row + c, cols - c);
    }
}

__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
    u32x4 q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<u32x4_a2*>(p) = q;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    u32x4 a, b;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = f_bits(v[j]), b[j] = f_bits(v[j + 4]);
    *reinterpret_cast<u32x4_a4*>(p) = a;
    *reinterpret_cast<u32x4_a4*>(p + 4) = b;
}
__device__ __forceinline__ void store8_nt(bf16* p, const float (&v)[8]) {
    u32x4 q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
    __builtin_nontemporal_store(q, reinterpret_cast<u32x4_a2*>(p));
}
__device__ __forceinline__ void store8_nt(float* p, const float (&v)[8]) { store8(p, v); }
template <bool NT = false, typename T>
__device__ __forceinline__ void store_chunk(T* row, int c, int cols, const float (&v)[8]) {
    if (c + 8 <= cols) {
        if (NT)
            store8_nt(row + c, v);
        else
            store8(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < cols) put(row + c + j, v[j]);
    }
}

// ---------------------------------------------------------------- lanes
// DPP moves inside rows of 16 lanes: quad_perm xor 1, xor 2, then mirrors, which exchange halves of
// 8 and of 16 lanes once every lane of a half holds the same value.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Largest value over aligned groups of 2^lb lanes (1 to 4; uniform).
__device__ __forceinline__ uint32_t group_max(uint32_t v, int lb) {
    v = umax(v, dpp<kDppXor1>(v));
    if (lb >= 2) v = umax(v, dpp<kDppXor2>(v));
    if (lb >= 3) v = umax(v, dpp<kDppHalfMirror>(v));
    if (lb >= 4) v = umax(v, dpp<kDppMirror>(v));
    return v;
}

// Sum over the wavefront, the same in every lane and in a fixed order.
__device__ __forceinline__ float wave_sum(float v) {
    v += bits_f(dpp<kDppXor1>(f_bits(v)));
    v += bits_f(dpp<kDppXor2>(f_bits(v)));
    v += bits_f(dpp<kDppHalfMirror>(f_bits(v)));
    v += bits_f(dpp<kDppMirror>(f_bits(v)));
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}

// ------------------------------------------------------------------ E8
// Largest magnitude of 8 values, as bits (NaN above infinity above the rest).
__device__ __forceinline__ uint32_t max_bits(const float (&v)[8]) {
    uint32_t m = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = umax(m, f_bits(v[j]) & 0x7fffffffu);
    return m;
}
// The exponent byte of a block from its largest magnitude's bits.
__device__ __forceinline__ uint32_t e8_exp(uint32_t bits) {
    const uint32_t f = bits >> 23;
    return f == 255u ? 255u : f > 7u ? f - 6u : 1u;
}
// 8 codes. The product x 2^(127 - E) is exact (or far below a half) and at most 128 in magnitude; adding 1.5 * 2^23 in
// the same instruction rounds it to an integer, ties to even, whose two's complement is the low byte. E = 255
// (where the products mean nothing) gives codes 0.
__device__ __forceinline__ u32x2 e8_encode(const float (&v)[8], uint32_t e) {
    constexpr float kMagic = 12582912.0f;
    const float inv = bits_f((254u - e) << 23);
    uint32_t t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        t[j] = f_bits(__builtin_amdgcn_fmed3f(__builtin_fmaf(v[j], inv, kMagic), kMagic - 127.0f, kMagic + 127.0f));
    const uint32_t keep = e == 255u ? 0u : ~0u;
    u32x2 q;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t lo = __builtin_amdgcn_perm(t[4 * j + 1], t[4 * j], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(t[4 * j + 3], t[4 * j + 2], 0x04000c0cu);
        q[j] = (lo | hi) & keep;
    }
    return q;
}
// The 8 values that codes stand for. scale = 2^(E - 127), infinite at E = 255 (codes 0: NaN).
// The product is exact: 7 bits and a sign, times a power of two.
__device__ __forceinline__ void e8_decode(u32x2 q, uint32_t e, float (&v)[8]) {
    const float s = bits_f(e << 23);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * j + i] = (float)((int32_t)(q[j] << (24 - 8 * i)) >> 24) * s;
    }
}

// Workgroups (w of n) go to the 8 XCDs in turn; this gives each XCD a contiguous eighth of the work, so that lines which
// neighbouring workgroups share (exponent bytes, row ends) stay in one L2.
__device__ __forceinline__ uint32_t xcd_block(uint32_t w, uint32_t n) {
    const uint32_t x = w & 7u, per = n >> 3, rest = n & 7u;
    return x * per + (x < rest ? x : rest) + (w >> 3);
}

// Quotient by a fixed divisor d >= 1 of n < 2^31: (n + mulhi(n, m)) >> l.
struct FastDiv {
    uint32_t d, m, l;
};
inline FastDiv fast_div(uint32_t d) {
    FastDiv f{d, 0, 0};
    while ((uint64_t(1) << f.l) < d) ++f.l;
    f.m = (uint32_t)((((uint64_t(1) << f.l) - d) << 32) / d + 1);
    return f;
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const FastDiv& f) {
    return (__umulhi(n, f.m) + n) >> f.l;
}

}  // namespace al
