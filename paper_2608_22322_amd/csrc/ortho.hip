// Orthogonalised updates: Newton-Schulz products of 16-bit parts on the matrix cores, and the momentum step around them.
//
// X0 = G / (|G| + eps) in the Frobenius norm, then X <- a X + (b A + c A A) X with A = X X^T, or for more rows than columns
// X <- a X + X (b A + c A A) with A = X^T X. A and A A are symmetric: the tiles below the diagonal are computed and written twice.
//
// Held between the products as fp16, scaled by powers of two, either one number (11 bits) or the sum of two (22 bits; the
// products hi hi + hi lo + lo hi). bf16 at the same speed has 8 bits: the products amplify what is lost in X by up to a^steps in
// directions of small singular values, and the result is 1e-2 off instead of 1.4e-3 (normal matrices). X0 is scaled by a power of two alone, so a bf16 G
// is held exactly; 1 / |G| goes into the sums of the first step.
#include <algorithm>
#include <cmath>

#include "mm_device.hpp"
#include "ortho_internal.hpp"

namespace al {

namespace {

typedef _Float16 f16;
typedef f16 f16x4 __attribute__((ext_vector_type(4)));

// X and A are held times 2^10, B = b A + c A A times 2^8. Singular values stay below 4 and those of B below 128 (the C ABI checks
// the coefficients), and the largest fp16 number is 65504; the elements of a 4096 x 11008 X0 are near 2^-13.
constexpr float kXScale = 1024.0f, kAScale = 1024.0f, kBScale = 256.0f;

struct Norm {
    double scale;  // 2^k with |G| + eps = nu 2^-k, nu in [1/2, 1)
    float inv, inv2;  // 1 / nu, 1 / nu^2
};

// Sum of squares of a matrix's slab, binary64 and in a fixed order.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[4];
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void square_kernel(const T* x, int64_t ld, int64_t rows, int cols, double* sums) {
    const int chunks = (cols + 7) / 8;
    const int64_t total = rows * chunks, per = (total + gridDim.x - 1) / gridDim.x, c0 = per * blockIdx.x, c1 = min(c0 + per, total);
    double s = 0;
    for (int64_t i = c0 + threadIdx.x; i < c1; i += 256) {
        const int64_t r = i / chunks;
        const int c = (int)(i - r * chunks) * 8;
        Chunk<T> k;
        load_chunk(k, x + r * ld, c, cols);
        float v[8];
        k.get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j] * (double)v[j];
    }
    s = block_sum(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// The norm of each matrix from its partial sums. A zero matrix gives zeros, one with an infinity or a NaN gives NaN.
__global__ __launch_bounds__(64) void norm_kernel(const double* sums, int count, double eps, Norm* norm) {
    const double* const p = sums + (int64_t)blockIdx.x * count;
    double s = 0;
    for (int i = threadIdx.x; i < count; i += 64) s += p[i];
    for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
    if (threadIdx.x) return;
    const double n = sqrt(s) + eps;
    Norm r;
    if (!(n < __builtin_inf())) {
        r.scale = 1.0;
        r.inv = r.inv2 = __builtin_nanf("");
    } else if (n == 0.0) {
        r.scale = 0.0;
        r.inv = r.inv2 = 0.0f;
    } else {
        int e;
        const double f = frexp(n, &e);
        r.scale = ldexp(1.0, -e);
        r.inv = (float)(1.0 / f);
        r.inv2 = (float)(1.0 / (f * f));
    }
    norm[blockIdx.x] = r;
}

__device__ __forceinline__ uint32_t pair(f16 a, f16 b) {
    return (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
}

// x (fp32 or bf16) -> X0 2^10 as one or two fp16 parts, padded with zeros. 8 columns a lane.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* x, int64_t ld, int64_t batch, int rows, int cols, int rp, int cp, int parts, const Norm* norm,
                                                   uint16_t* out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int chunks = cp / 8;
    if (i >= (int64_t)rp * chunks) return;
    const int r = (int)(i / chunks), c = (int)(i - (int64_t)r * chunks) * 8, b = blockIdx.y;
    float v[8] = {};
    if (r < rows) {
        Chunk<T> k;
        load_chunk(k, x + b * batch + r * ld, c, cols);
        k.get(v);
    }
    const double s = norm[b].scale * (double)kXScale;
    u32x4 hi, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f16 h[2], l[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float y = (float)((double)v[2 * j + e] * s);
            h[e] = (f16)y;
            l[e] = (f16)(y - (float)h[e]);
        }
        hi[j] = pair(h[0], h[1]);
        lo[j] = pair(l[0], l[1]);
    }
    const int64_t size = (int64_t)rp * cp;
    uint16_t* const o = out + b * parts * size + (int64_t)r * cp + c;
    *reinterpret_cast<u32x4*>(o) = hi;
    if (parts > 1) *reinterpret_cast<u32x4*>(o + size) = lo;
}

// A matrix of the workspace: size = side times side, the low part behind the high one.
struct Held {
    uint16_t* p;
    int64_t size;
    int32_t ld, parts;
    __device__ __forceinline__ f32x4 get(int b, int m, int n) const {
        const uint16_t* const q = p + b * parts * size + (int64_t)m * ld + n;
        f32x4 v = __builtin_convertvector(*reinterpret_cast<const f16x4*>(q), f32x4);
        if (parts > 1) v += __builtin_convertvector(*reinterpret_cast<const f16x4*>(q + size), f32x4);
        return v;
    }
    __device__ __forceinline__ void put(int b, int m, int n, f32x4 v, bool mirror) const {
        const f16x4 h = __builtin_convertvector(v, f16x4), l = __builtin_convertvector(v - __builtin_convertvector(h, f32x4), f16x4);
        uint16_t* const q = p + b * parts * size;
        *reinterpret_cast<f16x4*>(q + (int64_t)m * ld + n) = h;
        if (parts > 1) *reinterpret_cast<f16x4*>(q + size + (int64_t)m * ld + n) = l;
        if (mirror) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                *reinterpret_cast<f16*>(q + (int64_t)(n + r) * ld + m) = h[r];
                if (parts > 1) *reinterpret_cast<f16*>(q + size + (int64_t)(n + r) * ld + m) = l[r];
            }
        }
    }
};

// A = X X^T.
struct EndGram {
    Held a;
    const Norm* norm;  // first step: A = X0 X0^T / nu^2
    __device__ __forceinline__ void operator()(int b, int m, int n, f32x4 v, bool mirror) const {
        if (m >= a.ld || n >= a.ld) return;
        float s = kAScale / (kXScale * kXScale);
        if (norm) s *= norm[b].inv2;
        a.put(b, m, n, v * s, mirror);
    }
};

// B = b A + c A A.
struct EndPoly {
    Held a, o;
    float cb, cc;
    __device__ __forceinline__ void operator()(int b, int m, int n, f32x4 v, bool mirror) const {
        if (m >= a.ld || n >= a.ld) return;
        o.put(b, m, n, a.get(b, m, n) * (cb * (kBScale / kAScale)) + v * (cc * (kBScale / (kAScale * kAScale))), mirror);
    }
};

// X <- a X + B X: the next X, the result, or a step of the parameters.
struct EndBase {
    Held x;
    const Norm* norm;
    float ca;
    int32_t rows, cols;  // of the output
    __device__ __forceinline__ f32x4 next(int b, int m, int n, f32x4 v) const {
        v = x.get(b, m, n) * ca + v * (1.0f / kBScale);
        if (norm) v *= norm[b].inv;
        return v;
    }
};
struct EndNext : EndBase {
    Held o;
    __device__ __forceinline__ void operator()(int b, int m, int n, f32x4 v, bool) const {
        if (m < rows && n < cols) o.put(b, m, n, next(b, m, n, v), false);
    }
};
struct EndOut : EndBase {
    void* out;
    int64_t ld;
    int32_t out_bf16;
    __device__ __forceinline__ void operator()(int b, int m, int n, f32x4 v, bool) const {
        if (m >= rows || n >= cols) return;
        v = next(b, m, n, v) * (1.0f / kXScale);
        const int64_t i = m * ld + n;
        const int in = min(4, cols - n);
        if (out_bf16) {
            bf16* const p = static_cast<bf16*>(out) + i;
            typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
            if (in == 4) {
                *reinterpret_cast<u32x2_a2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                return;
            }
#pragma unroll
            for (int r = 0; r < 3; ++r)
                if (r < in) al::put(p + r, v[r]);
        } else {
            float* const p = static_cast<float*>(out) + i;
            typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
            if (in == 4) {
                *reinterpret_cast<f32x4_a4*>(p) = v;
                return;
            }
#pragma unroll
            for (int r = 0; r < 3; ++r)
                if (r < in) p[r] = v[r];
        }
    }
};
struct EndStep : EndBase {
    float* p[kMuonBatch];
    double decay, step;
    __device__ __forceinline__ void operator()(int b, int m, int n, f32x4 v, bool) const {
        if (m >= rows || n >= cols) return;
        v = next(b, m, n, v) * (1.0f / kXScale);
        float* const q = p[b] + (int64_t)m * cols + n;
        const int in = min(4, cols - n);
        typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
        if (in == 4) {
            f32x4 o = *reinterpret_cast<const f32x4_a4*>(q);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = (float)((double)o[r] * decay - step * (double)v[r]);
            *reinterpret_cast<f32x4_a4*>(q) = o;
            return;
        }
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < in) q[r] = (float)((double)q[r] * decay - step * (double)v[r]);
    }
};

template <bool AK, bool BK, class E>
hipError_t product(const MmCut& cut, Mm p, const E& end, hipStream_t st) {
    p.splits = cut.splits;
    if (cut.tile == 256) return mm_launch<f16, 256, AK, BK, false>(p, end, st);
    if (cut.tile == 128) return mm_launch<f16, 128, AK, BK, false>(p, end, st);
    return mm_launch<f16, 64, AK, BK, false>(p, end, st);
}

// The products of a batch whose X0 lies at x1; the last step's outputs go to `last`.
template <class E>
hipError_t iterate(const OrthoPlan& p, const OrthoCoefs& k, E last, char* ws, hipStream_t st) {
    const int64_t xs = (int64_t)p.rp * p.cp, ds = (int64_t)p.dp * p.dp;
    const Norm* const norm = reinterpret_cast<const Norm*>(ws + p.norm_off);
    Held x[2] = {{reinterpret_cast<uint16_t*>(ws + p.x1_off), xs, p.cp, p.parts}, {reinterpret_cast<uint16_t*>(ws + p.x0_off), xs, p.cp, p.parts}};
    const Held a = {reinterpret_cast<uint16_t*>(ws + p.a_off), ds, p.dp, p.parts}, b = {reinterpret_cast<uint16_t*>(ws + p.b_off), ds, p.dp, p.parts};
    const auto operand = [&](const Held& h, int rows) { return MmOperand{h.p, h.parts * h.size, h.size, h.ld, rows, h.ld}; };
    Mm q = {};
    q.segs = p.parts == 1 ? 1 : 3;
    q.amask = p.parts == 1 ? 0u : 4u;
    q.bmask = p.parts == 1 ? 0u : 2u;
    q.batches = p.batches;
    q.part = reinterpret_cast<float*>(ws + p.part_off);
    for (int i = 0; i < k.steps; ++i) {
        const Held &from = x[i & 1], &to = x[(i & 1) ^ 1];
        const Norm* const first = i == 0 ? norm : nullptr;
        const MmOperand ox = operand(from, p.rp), oa = operand(a, p.dp), ob = operand(b, p.dp);
        hipError_t e;
        Mm g = q;
        g.a = g.b = ox;
        g.m = g.n = p.dp;
        g.turns = (p.tall ? p.rp : p.cp) / kMmTurn;
        g.sym = 1;
        const EndGram gram = {a, first};
        if ((e = p.tall ? product<false, false>(p.g1, g, gram, st) : product<true, true>(p.g1, g, gram, st)) != hipSuccess) return e;
        g.a = g.b = oa;
        g.turns = p.dp / kMmTurn;
        const EndPoly poly = {a, b, k.b, k.c};
        if ((e = product<true, true>(p.g2, g, poly, st)) != hipSuccess) return e;
        g.sym = 0;
        g.m = p.rp;
        g.n = p.cp;
        g.a = p.tall ? ox : ob;
        g.b = p.tall ? ob : ox;
        const auto third = [&](auto end) {
            end.x = from;
            end.norm = first;
            end.ca = k.a;
            return p.tall ? product<true, true>(p.g3, g, end, st) : product<true, false>(p.g3, g, end, st);
        };
        if (i + 1 < k.steps) {
            EndNext next;
            next.rows = p.rp;
            next.cols = p.cp;
            next.o = to;
            e = third(next);
        } else {
            last.rows = (int32_t)p.rows;
            last.cols = (int32_t)p.cols;
            e = third(last);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
void pack(const OrthoPlan& p, const T* x, int64_t ld, int64_t batch, char* ws, hipStream_t st) {
    const dim3 grid((uint32_t)(((int64_t)p.rp * p.cp / 8 + 255) / 256), (uint32_t)p.batches);
    pack_kernel<T><<<grid, 256, 0, st>>>(x, ld, batch, (int)p.rows, (int)p.cols, p.rp, p.cp, p.parts, reinterpret_cast<const Norm*>(ws + p.norm_off),
                                         reinterpret_cast<uint16_t*>(ws + p.x1_off));
}

}  // namespace

MmCut mm_cut(int64_t m, int64_t n, int64_t turns, int64_t batches, bool sym) {
    static constexpr struct {
        int tile, fit;
        double ends, alone, each;
    } kinds[] = {{64, 4, 2, 0.45, 0.16}, {128, 2, 2, 0.8, 0.55}, {256, 1, 3, 2.0, 2.0}};
    static constexpr int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    MmCut best = {64, 1};
    double least = 0;
    for (const auto& k : kinds) {
        const int64_t s = (m + k.tile - 1) / k.tile, tiles = (sym ? s * (s + 1) / 2 : s * ((n + k.tile - 1) / k.tile)) * batches;
        for (const int c : counts) {
            if (c > 1 && (4 * c > turns || tiles * c > 1024)) break;
            const double load = (double)(tiles * c) / 256, whole = std::ceil(load), turn = k.fit == 1 ? k.each * whole : load > k.fit ? k.each * load : std::max(k.alone, k.each * whole),
                         t = ((double)((turns + c - 1) / c) + k.ends) * turn + (c > 1 ? 3 + 8e-7 * (double)(c * tiles) * k.tile * k.tile : 0);
            if (least == 0 || t < least) least = t, best = {k.tile, c};
        }
    }
    return best;
}

size_t mm_part_bytes(const MmCut& c, int64_t m, int64_t n, int64_t batches, bool sym) {
    if (c.splits == 1) return 0;
    const int64_t s = (m + c.tile - 1) / c.tile, tiles = sym ? s * (s + 1) / 2 : s * ((n + c.tile - 1) / c.tile);
    return (size_t)(tiles * batches * c.splits) * c.tile * c.tile * 4;
}

OrthoPlan ortho_plan(int64_t rows, int64_t cols, int32_t parts, int32_t batches, bool update) {
    OrthoPlan p = {};
    p.rows = rows;
    p.cols = cols;
    p.parts = parts;
    p.batches = batches;
    p.tall = rows > cols;
    p.rp = (int32_t)((rows + 63) / 64 * 64);
    p.cp = (int32_t)((cols + 63) / 64 * 64);
    p.dp = std::min(p.rp, p.cp);
    const int segs = parts == 1 ? 1 : 3;
    const int64_t kd = (int64_t)p.dp / kMmTurn * segs, kx = (int64_t)(p.tall ? p.rp : p.cp) / kMmTurn * segs;
    p.g1 = mm_cut(p.dp, p.dp, kx, batches, true);
    p.g2 = mm_cut(p.dp, p.dp, kd, batches, true);
    p.g3 = mm_cut(p.rp, p.cp, kd, batches, false);
    p.sums = (int32_t)(update ? (rows * cols + kMomentum - 1) / kMomentum : std::min<int64_t>(1024, (rows * cols + 4095) / 4096));
    const auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
    const size_t xs = (size_t)p.rp * p.cp, ds = (size_t)p.dp * p.dp;
    size_t off = 0;
    const auto take = [&](size_t bytes) {
        const size_t at = off;
        off += up(bytes);
        return at;
    };
    p.norm_off = take((size_t)batches * sizeof(Norm));
    p.sum_off = take((size_t)batches * p.sums * 8);
    p.x0_off = take(batches * xs * std::max(update ? 4 : 2, 2 * parts));
    p.x1_off = take(batches * xs * 2 * parts);
    p.a_off = take(batches * ds * 2 * parts);
    p.b_off = take(batches * ds * 2 * parts);
    p.part_off = take(std::max({mm_part_bytes(p.g1, p.dp, p.dp, batches, true), mm_part_bytes(p.g2, p.dp, p.dp, batches, true),
                                mm_part_bytes(p.g3, p.rp, p.cp, batches, false)}));
    p.bytes = off;
    return p;
}

hipError_t launch_orthogonalize(const OrthoPlan& p, const OrthoCoefs& k, int dtype, const void* x, int64_t ldx, int out_dtype, void* out, int64_t ldout,
                                void* ws, hipStream_t st) {
    char* const w = static_cast<char*>(ws);
    double* const sums = reinterpret_cast<double*>(w + p.sum_off);
    if (dtype == AL_DTYPE_BF16)
        square_kernel<bf16><<<p.sums, 256, 0, st>>>(static_cast<const bf16*>(x), ldx, p.rows, (int)p.cols, sums);
    else
        square_kernel<float><<<p.sums, 256, 0, st>>>(static_cast<const float*>(x), ldx, p.rows, (int)p.cols, sums);
    norm_kernel<<<1, 64, 0, st>>>(sums, p.sums, k.eps, reinterpret_cast<Norm*>(w + p.norm_off));
    if (dtype == AL_DTYPE_BF16)
        pack(p, static_cast<const bf16*>(x), ldx, 0, w, st);
    else
        pack(p, static_cast<const float*>(x), ldx, 0, w, st);
    EndOut last;
    last.out = out;
    last.ld = ldout;
    last.out_bf16 = out_dtype == AL_DTYPE_BF16;
    return iterate(p, k, last, w, st);
}

hipError_t launch_muon(const OrthoPlan& p, const OrthoCoefs& k, const MuonArgs& a, const MuonList& l, void* ws, hipStream_t st) {
    char* const w = static_cast<char*>(ws);
    double* const sums = reinterpret_cast<double*>(w + p.sum_off);
    float* const u = reinterpret_cast<float*>(w + p.x0_off);
    const int64_t n = p.rows * p.cols, pitch = (int64_t)p.rp * p.cp;
    const hipError_t e = launch_momentum(a, l, n, pitch, p.sums, p.batches, u, sums, st);
    if (e != hipSuccess) return e;
    norm_kernel<<<p.batches, 64, 0, st>>>(sums, p.sums, k.eps, reinterpret_cast<Norm*>(w + p.norm_off));
    pack(p, static_cast<const float*>(u), p.cols, pitch, w, st);
    EndStep last;
    for (int i = 0; i < kMuonBatch; ++i) last.p[i] = l.t[i].p;
    last.decay = a.decay;
    last.step = a.step;
    return iterate(p, k, last, w, st);
}

}  // namespace al
