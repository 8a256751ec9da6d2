// Orthogonalised updates: Newton-Schulz products of 16-bit parts on the matrix cores.
//
// X0 = G / (|G| + eps) in the Frobenius norm, then X <- a X + (b A + c A A) X with A = X X^T, or for more rows than columns
// X <- a X + X (b A + c A A) with A = X^T X. A and A A are symmetric: the tiles on and below the diagonal are computed and written twice.
//
// Held between the products as fp16, scaled by powers of two, either one number (11 bits) or the sum of two (22 bits; the
// products hi hi + hi lo + lo hi). bf16 at the same speed has 8 bits: the products amplify what is lost in X by up to a^steps in
// directions of small singular values, and the result is 1e-2 off instead of 1.4e-3 (normal matrices). X0 is scaled by a power of two alone, so a bf16 G's elements
// down to 2^-27 of its norm are held exactly; 1 / |G| goes into the sums of the first step. (fp16 ends at 2^-24: nothing is held closer than 2^-35 of X's norm, and two parts have all 22 bits of
// elements from 2^-13 of it on.)
//
// A step is three launches for all the matrices of a group (two where they are narrow, seven for two steps at once). Where whole tiles would leave compute units idle (136
// tiles for 256 of them, or matrices of different sizes), the group's turns are dealt out evenly instead: a workgroup takes a stretch of them, across tiles, and tiles
// that two or more worked on are joined in a second launch, in order; or the tiles behind the last full round are taken in pieces.
//
// Bound by the matrix cores where matrices are large: 4096 x 11008 in one part 2.77 to 2.86 ms, 1.0 to 1.2 PFLOP/s in its products (a library product of 4096^3 1.38); by
// launches and by what one or two workgroups a compute unit reach where they are not: 1001 x 1750 in two parts 285 us, 1.0e11 operations.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "mm_cut.hpp"
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
    double scale;     // 2^k with |G| + eps = nu 2^-k, nu in [1/2, 1)
    float inv, inv2;  // 1 / nu, 1 / nu^2
};

// The workgroup's sum, in a fixed order.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[4];
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// Sums of squares of a matrix's slabs.
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

// The norm of a matrix from its partial sums, by a workgroup. A zero matrix gives zeros, one with an infinity or a NaN gives NaN.
__device__ __forceinline__ Norm norm_of(const double* sums, uint32_t count, double eps) {
    double s = 0;
    for (uint32_t i = threadIdx.x; i < count; i += 256) s += sums[i];
    const double n = sqrt(block_sum(s)) + eps;
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
    return r;
}

__device__ __forceinline__ uint32_t pair(f16 a, f16 b) {
    return (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
}

// Partial sums of a matrix that every workgroup of pack_kernel adds up for itself: there is one of these for 2048 elements, and al_muon_step leaves a sum for 8192, so that what is read grows with
// the square of the size (2^21 x 512: 30 ms of a step's 37). More are added up in a launch before.
constexpr uint32_t kMostSums = 1024;

struct PackList {
    struct {
        const void* x;
        int64_t ld;
        uint16_t* out;
        int32_t rows, cols, rp, cp;
    } t[kOrthoGroup];
    uint32_t begin[kOrthoGroup + 1];  // workgroups (2048 elements each)
    uint32_t sums[kOrthoGroup + 1];   // partial sums of squares
    int32_t count;
};

// The norms of the matrices with many partial sums, a workgroup each.
__global__ __launch_bounds__(256) void norm_kernel(PackList l, double eps, const double* sums, Norm* norms) {
    const uint32_t b = blockIdx.x, n = l.sums[b + 1] - l.sums[b];
    if (n <= kMostSums) return;
    const Norm norm = norm_of(sums + l.sums[b], n, eps);
    if (threadIdx.x == 0) norms[b] = norm;
}

// x (fp32 or bf16) -> X0 2^10 as one or two fp16 parts, padded with zeros: 8 columns a lane. Each workgroup takes the norm from up to kMostSums partial sums by itself (a launch
// less); the first of a matrix writes it for the first step's sums.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackList l, int parts, double eps, const double* sums, Norm* norms) {
    int b = 0;
    while (b + 1 < l.count && blockIdx.x >= l.begin[b + 1]) ++b;
    const auto& t = l.t[b];
    const uint32_t n = l.sums[b + 1] - l.sums[b];
    const Norm norm = n > kMostSums ? norms[b] : norm_of(sums + l.sums[b], n, eps);
    if (n <= kMostSums && threadIdx.x == 0 && blockIdx.x == l.begin[b]) norms[b] = norm;
    const int64_t i = (int64_t)(blockIdx.x - l.begin[b]) * 256 + threadIdx.x;
    const int chunks = t.cp / 8, r = (int)(i / chunks), c = (int)(i - (int64_t)r * chunks) * 8;
    float v[8] = {};
    if (r < t.rows) {
        Chunk<T> k;
        load_chunk(k, static_cast<const T*>(t.x) + r * t.ld, c, t.cols);
        k.get(v);
    }
    const double s = norm.scale * (double)kXScale;
    u32x4 hi, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f16 h[2], w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float y = (float)((double)v[2 * j + e] * s);
            h[e] = (f16)y;
            w[e] = (f16)(y - (float)h[e]);
        }
        hi[j] = pair(h[0], h[1]);
        lo[j] = pair(w[0], w[1]);
    }
    uint16_t* const o = t.out + (int64_t)r * t.cp + c;
    *reinterpret_cast<u32x4*>(o) = hi;
    if (parts > 1) *reinterpret_cast<u32x4*>(o + (int64_t)t.rp * t.cp) = lo;
}

// A matrix of the workspace, the low part behind the high one.
struct Held {
    uint16_t* p;
    int64_t size;
    int32_t ld, parts;
    __device__ __forceinline__ f32x4 get(int m, int n) const {
        const uint16_t* const q = p + (int64_t)m * ld + n;
        f32x4 v = __builtin_convertvector(*reinterpret_cast<const f16x4*>(q), f32x4);
        if (parts > 1) v += __builtin_convertvector(*reinterpret_cast<const f16x4*>(q + size), f32x4);
        return v;
    }
    __device__ __forceinline__ void put(int m, int n, f32x4 v, bool mirror) const {
        const f16x4 h = __builtin_convertvector(v, f16x4), l = __builtin_convertvector(v - __builtin_convertvector(h, f32x4), f16x4);
        *reinterpret_cast<f16x4*>(p + (int64_t)m * ld + n) = h;
        if (parts > 1) *reinterpret_cast<f16x4*>(p + size + (int64_t)m * ld + n) = l;
        if (mirror) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                *reinterpret_cast<f16*>(p + (int64_t)(n + r) * ld + m) = h[r];
                if (parts > 1) *reinterpret_cast<f16*>(p + size + (int64_t)(n + r) * ld + m) = l[r];
            }
        }
    }
    __device__ __forceinline__ MmOperand operand(int rows) const { return {p, size, ld, rows, ld}; }
};

// The products of a step: A = X X^T, B = b A + c A A, and a X + B X as the next X, the result, or a step of the parameters.
//
// Two steps at once: what multiplies X is a polynomial of A, and so is the next step's A. With M = a I + B, which commutes with A,
//   A' = M A M,  B' = b A' + c A' A',  X'' = (a I + B') M X = a a X + D X,  D = a B + a B' + B' B:
// the next step's A by Y = M A = a A + B A and A' = Y M = a Y + Y B, and no X in between. Three more products of symmetric matrices (half of each is
// computed) for one of X with its transpose and one with X, which is less work where X is long. Each pair starts anew from its X: in fp16 parts the singular
// values that A holds badly, those far below the largest, grow by 3.4 a step, and over two steps that costs little (two parts, 1024 x 2816: 3.3e-6 for 3.1e-6 off in
// the Frobenius norm; three steps 5.6e-6, five on values falling as 1 / k 1e-4).
enum Kind : int { kGram, kPoly, kNext, kOut, kStep };

// A product of two symmetric matrices of an item: out = sum factor + one c1 + two c2 (c2 = 0: without). The numbers are the matrices' places.
struct Square {
    int32_t a, b, one, two, out;
    float factor, c1, c2;
};
__host__ __device__ constexpr bool square_kind(int kind) { return kind == kGram || kind == kPoly; }

struct OrthoLaunch {
    OrthoItem it[kOrthoGroup];
    int64_t begin[kOrthoGroup + 1];  // first tile of each item, or, with slots, first turn
    int64_t slots;                   // workgroups that the turns are dealt out to; 0: a tile a workgroup, or a piece of one:
    uint32_t whole;                  // tiles that are taken whole
    uint32_t rest, split;            // the tiles behind them, each in so many pieces
    int32_t count, parts, from, first;  // from: which place X is in; first: the first step
    int32_t by;                          // which square matrix X is multiplied with, and
    float ca;                            // the multiple of X that is added
    Square square;
    const Norm* norms;
    float* part;  // [2 slots][a tile in the lanes' order]
    double decay;
    void* out;
    int64_t ldout;
    int32_t out_bf16;
};

__host__ __device__ inline int64_t item_tiles(const OrthoItem& t, int kind, int tile) {
    if (!square_kind(kind)) return (int64_t)((t.rp + tile - 1) / tile) * ((t.cp + tile - 1) / tile);
    const int64_t s = ((t.rp < t.cp ? t.rp : t.cp) + tile - 1) / tile;
    return s * (s + 1) / 2;
}
// Turns of a segment, and segments.
__host__ __device__ inline int32_t item_turns(const OrthoItem& t, int kind) {
    return (kind == kGram ? (t.rp > t.cp ? t.rp : t.cp) : t.rp < t.cp ? t.rp : t.cp) / kMmTurn;
}
__host__ __device__ constexpr int32_t item_segments(int tile, int parts) { return tile > 64 && parts > 1 ? 3 : 1; }

// One item's product.
template <int KIND>
struct Task {
    const OrthoLaunch& a;
    const OrthoItem t;
    int item;
    bool tall;
    int32_t dp, own;  // own: places from a launch's square matrices to this tile's
    Held x;
    // the item's square matrices
    __device__ __forceinline__ Held square(int i) const {
        const int64_t n = (int64_t)dp * dp;
        return {t.a + i * a.parts * n, n, dp, a.parts};
    }
    __device__ __forceinline__ Task(const OrthoLaunch& l, int i, int to = 0) : a(l), t(l.it[i]), item(i), own(to) {
        tall = t.rp > t.cp || (t.rp == t.cp && t.rows > t.cols);
        dp = min(t.rp, t.cp);
        x = {a.from ? t.x[1] : t.x[0], (int64_t)t.rp * t.cp, t.cp, a.parts};
    }
    template <int B>
    __device__ __forceinline__ Mm product() const {
        Mm p;
        p.segs = item_segments(B, a.parts);
        p.amask = p.segs > 1 ? 4u : 0u;
        p.bmask = p.segs > 1 ? 2u : 0u;
        p.splits = 1;
        p.part = nullptr;
        p.sym = square_kind(KIND);
        p.m = square_kind(KIND) ? dp : t.rp;
        p.n = square_kind(KIND) ? dp : t.cp;
        p.turns = item_turns(t, KIND);
        const MmOperand ox = x.operand(t.rp);
        p.a = KIND == kGram ? ox : KIND == kPoly ? square(a.square.a).operand(dp) : tall ? ox : square(a.by + own).operand(dp);
        p.b = KIND == kGram ? ox : KIND == kPoly ? square(a.square.b).operand(dp) : tall ? square(a.by + own).operand(dp) : ox;
        return p;
    }
    // What the product is combined with: sum * factor() + one() * other() + two() * second(), and that times after().
    __device__ __forceinline__ Held one() const { return KIND == kPoly ? square(a.square.one) : x; }
    __device__ __forceinline__ Held two() const { return square(a.square.two); }
    __device__ __forceinline__ float factor() const {
        return KIND == kGram ? kAScale / (kXScale * kXScale) * (a.first ? a.norms[item].inv2 : 1.0f) : KIND == kPoly ? a.square.factor : 1.0f / kBScale;
    }
    __device__ __forceinline__ float other() const { return KIND == kPoly ? a.square.c1 : a.ca; }
    __device__ __forceinline__ float second() const { return KIND == kPoly ? a.square.c2 : 0.0f; }
    __device__ __forceinline__ float after() const { return !square_kind(KIND) && a.first ? a.norms[item].inv : 1.0f; }
    // where it goes, for what stays in the workspace
    __device__ __forceinline__ Held to() const {
        if (KIND == kGram) return square(0);
        if (KIND == kPoly) return square(a.square.out + own);
        return {a.from ? t.x[0] : t.x[1], x.size, x.ld, a.parts};
    }
    __device__ __forceinline__ int32_t rows() const { return square_kind(KIND) ? dp : t.rp; }
    __device__ __forceinline__ int32_t cols() const { return square_kind(KIND) ? dp : t.cp; }

    // 4 neighbouring values of the result or of the parameters
    __device__ __forceinline__ void write(int m, int n, f32x4 v) const {
        if (m >= t.rows || n >= t.cols) return;
        v *= 1.0f / kXScale;
        const int in = min(4, t.cols - n);
        typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
        typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
        if constexpr (KIND == kStep) {
            float* const q = t.p + (int64_t)m * t.cols + n;
            if (in == 4) {
                f32x4 o = *reinterpret_cast<const f32x4_a4*>(q);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = (float)((double)o[r] * a.decay - t.step * (double)v[r]);
                *reinterpret_cast<f32x4_a4*>(q) = o;
            } else {
#pragma unroll
                for (int r = 0; r < 3; ++r)
                    if (r < in) q[r] = (float)((double)q[r] * a.decay - t.step * (double)v[r]);
            }
        } else if (a.out_bf16) {
            bf16* const q = static_cast<bf16*>(a.out) + m * a.ldout + n;
            if (in == 4) {
                *reinterpret_cast<u32x2_a2*>(q) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            } else {
#pragma unroll
                for (int r = 0; r < 3; ++r)
                    if (r < in) al::put(q + r, v[r]);
            }
        } else {
            float* const q = static_cast<float*>(a.out) + m * a.ldout + n;
            if (in == 4) {
                *reinterpret_cast<f32x4_a4*>(q) = v;
            } else {
#pragma unroll
                for (int r = 0; r < 3; ++r)
                    if (r < in) q[r] = v[r];
            }
        }
    }
    // 4 neighbouring outputs from their sums
    __device__ __forceinline__ void end(int m, int n, f32x4 v, bool mirror) const {
        if (m >= rows() || n >= cols()) return;
        v *= factor();
        if constexpr (KIND != kGram) v += one().get(m, n) * other();
        if (KIND == kPoly && second() != 0.0f) v += two().get(m, n) * second();
        v *= after();
        if constexpr (KIND == kOut || KIND == kStep)
            write(m, n, v);
        else
            to().put(m, n, v, mirror);
    }
};

// A tile of one part in LDS, in the places of the turns (64 rows in each): rows of B values whose 16-byte pieces are exchanged by the row, so that the lanes' quads
// (16 rows at once) and whole rows both meet all banks. The tile's ends go through it: the lanes' own 8-byte pieces of 16 rows at
// a time take 25 us of memory accesses for a 256 x 256 tile.
template <int B>
struct Image {
    typedef MmTile<B> G;
    static constexpr int kMask = B == 64 ? 7 : 15;
    typedef __attribute__((address_space(3))) uint16_t* lds_u16;
    typedef __attribute__((address_space(3))) u32x4* lds_u32x4;
    typedef __attribute__((address_space(3))) f16x4* lds_f16x4;
    typedef __attribute__((address_space(3))) f16* lds_f16;
    uint32_t a0, a1, b0, b1;  // LDS addresses (a choice among pointers would be a generic one)
    __device__ __forceinline__ Image(uint16_t* p0, uint16_t* p1, uint16_t* p2, uint16_t* p3)
        : a0((uint32_t)(uintptr_t)(lds_u16)p0), a1((uint32_t)(uintptr_t)(lds_u16)p1), b0((uint32_t)(uintptr_t)(lds_u16)p2),
          b1((uint32_t)(uintptr_t)(lds_u16)p3) {}
    // rows 64 q .. 64 q + 63
    __device__ __forceinline__ uint32_t rows(int q) const { return B == 64 ? a0 : B == 128 ? (q & 1 ? a1 : a0) : q & 2 ? (q & 1 ? b1 : b0) : (q & 1 ? a1 : a0); }
    // bytes from those on
    static __device__ __forceinline__ uint32_t offset(int row, int col) {
        return (uint32_t)((row & 63) * B + ((((col >> 3) ^ row) & kMask) << 3) + (B > 128 ? col & 128 : 0) + (col & 7)) * 2u;
    }
    __device__ __forceinline__ lds_u32x4 piece(int k) const {
        const int row = k / (B / 8), col = k % (B / 8) * 8;
        return (lds_u32x4)(uintptr_t)(rows(row >> 6) + offset(row, col));
    }
    // f(sums, their quad) for the lane's quads: row r + 16 i, columns c + 16 j ..
    template <class F>
    __device__ __forceinline__ void quads(int r, int c, MmAcc (&acc)[G::FM][G::FN], const F& f) const {
        uint32_t off = offset(r, c);
        asm volatile("" : "+v"(off));  // (32 addresses a pass would not stay in registers)
#pragma unroll
        for (int i = 0; i < G::FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            const uint32_t q = rows(__builtin_amdgcn_readfirstlane(r >> 6) + i / 4) + i % 4 * 32 * B;
#pragma unroll
            for (int j = 0; j < G::FN; ++j) f(acc[i][j], (lds_f16x4)(uintptr_t)(q + (off ^ (uint32_t)(j << 5))));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // the lane's quads across the diagonal: element e of a quad at row c + 16 j + e, column r + 16 i
    __device__ __forceinline__ void across(int r, int c, const MmAcc (&acc)[G::FM][G::FN]) const {
        uint32_t off[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            off[e] = offset(c + e, r);
            asm volatile("" : "+v"(off[e]));
        }
        const uint32_t q = rows(__builtin_amdgcn_readfirstlane(c >> 6));
#pragma unroll
        for (int i = 0; i < G::FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < G::FN; ++j) {
                const f16x4 h = __builtin_convertvector(acc[i][j], f16x4);
#pragma unroll
                for (int e = 0; e < 4; ++e) *(lds_f16)(uintptr_t)(q + j * 32 * B + (off[e] ^ (uint32_t)(i << 5))) = h[e];
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // Rows and columns m0, n0 .. of a matrix of m x n (multiples of 64): a thread takes one column of pieces, 4 rows of them at a time.
    static constexpr int kPer = B * B / 8 / G::kThreads, kStep = G::kThreads / (B / 8);
    __device__ __forceinline__ void load(int tid, const uint16_t* p, int ld, int m0, int n0, int m, int n) const {
        const int row = tid / (B / 8), col = tid % (B / 8) * 8;
        const bool in = n0 + col < n;
        const uint16_t* q = p + (int64_t)(m0 + row) * ld + n0 + col;
#pragma unroll 1
        for (int i = 0; i < kPer; i += 4) {
            u32x4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = 0u;
                if (i + j < kPer && in && m0 + row + (i + j) * kStep < m) v[j] = *reinterpret_cast<const u32x4*>(q);
                q += (int64_t)kStep * ld;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j < kPer) *piece((i + j) * G::kThreads + tid) = v[j];
        }
    }
    __device__ __forceinline__ void store(int tid, uint16_t* p, int ld, int m0, int n0, int m, int n) const {
        const int row = tid / (B / 8), col = tid % (B / 8) * 8;
        if (n0 + col >= n) return;
        uint16_t* q = p + (int64_t)(m0 + row) * ld + n0 + col;
#pragma unroll 1
        for (int i = 0; i < kPer; ++i, q += (int64_t)kStep * ld)
            if (m0 + row + i * kStep < m) *reinterpret_cast<u32x4*>(q) = *piece(i * G::kThreads + tid);
    }
};

// The end of a tile (m0, n0: its first row and column).
template <int B, int KIND>
__device__ __forceinline__ void finish(const Task<KIND>& task, int m0, int n0, const Image<B>& image, MmAcc (&acc)[MmTile<B>::FM][MmTile<B>::FN]) {
    typedef MmTile<B> G;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // (what follows from it is formed here, not carried through the products in registers that they need)
    const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = G::wave_m(w) + (lane & 15), c = G::wave_n(w) + 4 * (lane >> 4);  // the lane's first row and columns
    const auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < G::FM; ++i)
#pragma unroll
            for (int j = 0; j < G::FN; ++j) f(acc[i][j]);
    };
    // (keeps the compiler from holding on to one pass's conversions for the next)
    const auto renew = [&]() __attribute__((always_inline)) { each([&](f32x4& v) { asm volatile("" : "+v"(v)); }); };
    const float factor = task.factor(), other = task.other(), after = task.after();
    const int parts = task.a.parts, m = task.rows(), n = task.cols();
    each([&](f32x4& v) { v *= factor; });
    if constexpr (KIND != kGram) {
        const int32_t added = parts * (task.second() != 0.0f ? 2 : 1);
#pragma unroll 1
        for (int p = 0; p < added; ++p) {
            const bool first = p < parts;
            const Held f = first ? task.one() : task.two();
            const float by = first ? other : task.second();
            image.load(tid, f.p + (first ? p : p - parts) * f.size, f.ld, m0, n0, m, n);
            __syncthreads();
            image.quads(r, c, acc, [&](f32x4& v, auto q) { v += __builtin_convertvector((f16x4)*q, f32x4) * by; });
            __syncthreads();
        }
        each([&](f32x4& v) { v *= after; });
    }
    if constexpr (KIND == kOut || KIND == kStep) {
#pragma unroll
        for (int i = 0; i < G::FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < G::FN; ++j) task.write(m0 + r + 16 * i, n0 + c + 16 * j, acc[i][j]);
        }
    } else {
        const Held o = task.to();
#pragma unroll 1
        for (int p = 0; p < parts; ++p) {
            uint16_t* const q = o.p + p * o.size;
            image.quads(r, c, acc, [&](f32x4& v, auto q) { *q = __builtin_convertvector(v, f16x4); });
            __syncthreads();
            image.store(tid, q, o.ld, m0, n0, m, n);
            if (square_kind(KIND) && m0 != n0) {
                __syncthreads();
                renew();
                image.across(r, c, acc);
                __syncthreads();
                image.store(tid, q, o.ld, n0, m0, n, m);
            }
            if (p + 1 < parts) {
                __syncthreads();
                renew();
                each([&](f32x4& v) { v -= __builtin_convertvector(__builtin_convertvector(v, f16x4), f32x4); });
            }
        }
    }
}

// First turn of slot g of a launch whose turns are dealt out.
__device__ __forceinline__ int64_t slot_begin(const OrthoLaunch& a, int64_t g) { return g * a.begin[a.count] / a.slots; }
__device__ __forceinline__ int item_at(const OrthoLaunch& a, int64_t pos) {
    int i = 0;
    while (i + 1 < a.count && pos >= a.begin[i + 1]) ++i;
    return i;
}

// Turns t0 .. t1 of a tile, and its end or, where that is not all of it, its partial sums.
template <int B, int KIND, int PARTS>
using PlacesOf = MmPlaces<PARTS, PARTS, mm_stages<B, PARTS, PARTS>()>;
template <int B, int KIND, int PARTS, bool PIECE, bool TALL>
__device__ __forceinline__ void segment(const Task<KIND>& task, int tile, int t0, int t1, int64_t place, const PlacesOf<B, KIND, PARTS>& at) {
    typedef MmTile<B> G;
    const Mm p = task.template product<B>();
    const MmAt id = mm_at<B>(p, (uint32_t)tile);
    MmAcc acc[G::FM][G::FN] = {};
    constexpr bool kRows = KIND == kPoly || (KIND == kGram ? !TALL : true), kCols = KIND == kPoly || (KIND == kGram ? !TALL : TALL);  // k along the rows
    MmCore<f16, B, kRows, kCols, kMmWhole, PARTS, PARTS>::run(p, id.m * B, id.n * B, t0, t1, at, acc);
    if (PIECE || t1 - t0 < p.turns * p.segs) {
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        f32x4* const part = reinterpret_cast<f32x4*>(task.a.part) + (place * G::kWaves + w) * (G::FM * G::FN * 64) + lane;
#pragma unroll
        for (int r = 0; r < G::FM; ++r)
#pragma unroll
            for (int j = 0; j < G::FN; ++j) part[(r * G::FN + j) * 64] = acc[r][j];
    } else {
        __syncthreads();  // every wavefront has read its last turn
        finish<B, KIND>(task, id.m * B, id.n * B, Image<B>(at.a[0][0], at.a[1][0], at.b[0][0], at.b[1][0]), acc);
    }
}
template <int B, int KIND, int PARTS, bool PIECE = false>
__device__ __forceinline__ void segment(const Task<KIND>& task, int tile, int t0, int t1, int64_t place, const PlacesOf<B, KIND, PARTS>& at) {
    if (KIND != kPoly && task.tall)
        segment<B, KIND, PARTS, PIECE, true>(task, tile, t0, t1, place, at);
    else
        segment<B, KIND, PARTS, PIECE, false>(task, tile, t0, t1, place, at);
}

// An XCD takes a contiguous eighth of each item's tiles, the items one after the other (longest first): contiguous eighths of all the tiles would leave the long ones
// to some of the XCDs. Items with few tiles begin at different XCDs. False: no tile for this workgroup.
__device__ __forceinline__ bool whole_tile(const OrthoLaunch& a, int& i, uint32_t& tile) {
    uint32_t k = blockIdx.x >> 3;
    tile = 0;
    for (i = 0; i < a.count; ++i) {
        const uint32_t n = (uint32_t)(min(a.begin[i + 1], (int64_t)a.whole) - min(a.begin[i], (int64_t)a.whole)), x = (blockIdx.x + (uint32_t)i) & 7u, per = n >> 3,
                       rest = n & 7u, mine = per + (x < rest ? 1u : 0u);
        tile = x * per + min(x, rest) + k;
        if (k < mine) return true;
        k -= mine;
    }
    return false;
}

template <int B, int KIND, int PARTS>
__global__ __launch_bounds__(MmTile<B>::kThreads, 2) void ortho_kernel(OrthoLaunch a) {
    constexpr int PA = PARTS, PB = PARTS;
    MM_PLACES(B, PA, PB, places);
    int i;
    uint32_t tile;
    if (!whole_tile(a, i, tile)) return;
    segment<B, KIND, PARTS>(Task<KIND>(a, i), (int32_t)tile, 0, item_turns(a.it[i], KIND) * item_segments(B, a.parts), 0, places);
}

// Matrices with a shorter side of up to 64, whose b A + c A A is one tile: each workgroup of X's product takes it for itself, into a place of its own (500 x 64: 5
// launches less, 64 us of kernels in place of 75).
template <int KIND, int PARTS>
__global__ __launch_bounds__(MmTile<64>::kThreads, 2) void ortho_narrow_kernel(OrthoLaunch a) {
    constexpr int PA = PARTS, PB = PARTS;
    MM_PLACES(64, PA, PB, places);
    int i;
    uint32_t tile;
    if (!whole_tile(a, i, tile)) return;
    segment<64, kPoly, PARTS>(Task<kPoly>(a, i, (int)tile), 0, 0, 1, 0, places);
    __threadfence_block();  // the workgroup's stores of its own place before its loads
    __syncthreads();
    segment<64, KIND, PARTS>(Task<KIND>(a, i, (int)tile), (int32_t)tile, 0, 1, 0, places);
}

// The pieces of the tiles behind the whole ones, those at one place of k neighbours.
template <int B, int KIND, int PARTS>
__global__ __launch_bounds__(MmTile<B>::kThreads, 2) void ortho_pieces_kernel(OrthoLaunch a) {
    constexpr int PA = PARTS, PB = PARTS;
    MM_PLACES(B, PA, PB, places);
    const uint32_t piece = blockIdx.x / a.rest, tile = a.whole + blockIdx.x - piece * a.rest;
    const int i = item_at(a, tile);
    const uint64_t turns = (uint64_t)(item_turns(a.it[i], KIND) * item_segments(B, a.parts));
    segment<B, KIND, PARTS, true>(Task<KIND>(a, i), (int32_t)(tile - a.begin[i]), __builtin_amdgcn_readfirstlane((int32_t)(piece * turns / a.split)),
                                  __builtin_amdgcn_readfirstlane((int32_t)((piece + 1) * turns / a.split)), blockIdx.x, places);
}

// The turns dealt out to slots. (Kernels of their own: the loop over a slot's tiles takes registers that 256-wide tiles do not have.)
template <int B, int KIND, int PARTS>
__global__ __launch_bounds__(MmTile<B>::kThreads, 2) void ortho_slots_kernel(OrthoLaunch a) {
    constexpr int PA = PARTS, PB = PARTS;
    MM_PLACES(B, PA, PB, places);
    const int64_t g = xcd_block(blockIdx.x, gridDim.x), stop = slot_begin(a, g + 1);
    int64_t at = slot_begin(a, g), place = 2 * g;
    while (at < stop) {
        const int i = item_at(a, at);
        const Task<KIND> task(a, i);
        const int32_t turns = item_turns(a.it[i], KIND) * item_segments(B, a.parts);
        const int64_t local = at - a.begin[i];
        const int32_t tile = __builtin_amdgcn_readfirstlane((int32_t)(local / turns)), t0 = __builtin_amdgcn_readfirstlane((int32_t)(local - (int64_t)tile * turns)), t1 = (int32_t)min((int64_t)turns, t0 + (stop - at));
        segment<B, KIND, PARTS>(task, tile, t0, t1, place, places);
        at += t1 - t0;
        place = 2 * g + 1;
        __syncthreads();  // every wavefront has read its last turn, or the tile's last image
    }
}

// The tiles that slots share, each joined by the workgroups of the first slot that begins inside it.
template <int B, int KIND>
__global__ __launch_bounds__(256) void ortho_join_kernel(OrthoLaunch a) {
    typedef MmTile<B> G;
    constexpr uint32_t kBlocks = B * B / 1024;
    const int64_t g = blockIdx.x / kBlocks + 1, pos = slot_begin(a, g);
    const int i = item_at(a, pos);
    const Task<KIND> task(a, i);
    const Mm p = task.template product<B>();
    const int32_t turns = p.turns * p.segs, tile = (int32_t)((pos - a.begin[i]) / turns);
    const int64_t s = a.begin[i] + (int64_t)tile * turns, e = s + turns, before = slot_begin(a, g - 1);
    if (pos == s || before > s) return;
    const uint32_t at = blockIdx.x % kBlocks * 256 + threadIdx.x, lane = at & 63, slot = at >> 6;
    const f32x4* const part = reinterpret_cast<const f32x4*>(a.part) + at;
    constexpr int64_t kTile = B * B / 4;
    const int64_t last = (e * a.slots - 1) / a.begin[a.count];  // the last slot that begins before e
    f32x4 v = part[(2 * (g - 1) + (before < s ? 1 : 0)) * kTile];
    for (int64_t h = g; h <= last; h += 8) {
        f32x4 q[8];
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (h + r <= last) q[r] = part[2 * (h + r) * kTile];
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (h + r <= last) v += q[r];
    }
    const MmAt id = mm_at<B>(p, (uint32_t)tile);
    const uint32_t w = slot / (G::FM * G::FN), q = slot % (G::FM * G::FN);
    task.end(id.m * B + G::wave_m((int)w) + (int)(lane & 15) + 16 * (int)(q / G::FN), id.n * B + G::wave_n((int)w) + 4 * (int)(lane >> 4) + 16 * (int)(q % G::FN), v,
             p.sym && id.m != id.n);
}

// The tiles that were taken in pieces.
template <int B, int KIND>
__global__ __launch_bounds__(256) void ortho_sum_kernel(OrthoLaunch a) {
    typedef MmTile<B> G;
    constexpr uint32_t kBlocks = B * B / 1024;
    const uint32_t r = blockIdx.x / kBlocks;
    const int i = item_at(a, a.whole + r);
    const Task<KIND> task(a, i);
    const uint32_t at = blockIdx.x % kBlocks * 256 + threadIdx.x, lane = at & 63, slot = at >> 6;
    const f32x4* const part = reinterpret_cast<const f32x4*>(a.part) + at;
    constexpr int64_t kTile = B * B / 4;
    f32x4 v = {};
    for (uint32_t h = 0; h < a.split; h += 8) {
        f32x4 q[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (h + j < a.split) q[j] = part[((int64_t)(h + j) * a.rest + r) * kTile];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (h + j < a.split) v += q[j];
    }
    const Mm p = task.template product<B>();
    const MmAt id = mm_at<B>(p, (uint32_t)(a.whole + r - a.begin[i]));
    const uint32_t w = slot / (G::FM * G::FN), q = slot % (G::FM * G::FN);
    task.end(id.m * B + G::wave_m((int)w) + (int)(lane & 15) + 16 * (int)(q / G::FN), id.n * B + G::wave_n((int)w) + 4 * (int)(lane >> 4) + 16 * (int)(q % G::FN), v,
             p.sym && id.m != id.n);
}

template <int B, int KIND, int PARTS>
hipError_t launch(OrthoLaunch& a, hipStream_t st) {
    if constexpr (B < 256) {
        if (a.slots) {
            ortho_slots_kernel<B, KIND, PARTS><<<(uint32_t)a.slots, MmTile<B>::kThreads, 0, st>>>(a);
            ortho_join_kernel<B, KIND><<<(uint32_t)((a.slots - 1) * (B * B / 1024)), 256, 0, st>>>(a);
            return hipGetLastError();
        }
    }
    a.whole = (uint32_t)a.begin[a.count] - a.rest;
    uint32_t most = 0;  // of an XCD
    for (int i = 0; i < a.count; ++i) most += (uint32_t)((std::min<int64_t>(a.begin[i + 1], a.whole) - std::min<int64_t>(a.begin[i], a.whole) + 7) / 8);
    if (most) ortho_kernel<B, KIND, PARTS><<<8 * most, MmTile<B>::kThreads, 0, st>>>(a);
    if (a.rest) {
        ortho_pieces_kernel<B, KIND, PARTS><<<a.rest * a.split, MmTile<B>::kThreads, 0, st>>>(a);
        ortho_sum_kernel<B, KIND><<<a.rest * (B * B / 1024), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

// How a group's product is cut: the tile and, where that is faster by the measured times, the slots that its turns are dealt out to. Slots that work at different places of k
// share little of what they load: whole tiles run in step and find their neighbours' loads in the L2. What dealing out is for is few tiles and a long sum.
// Tiles of one length that are some rounds of the device and a few more: the rounds are taken whole, the rest in pieces, up to three rounds of them (4096 x 11008, A: 136
// tiles of 256, half of a round, 269 us, 528 of 128, of which 16 in 32 pieces each, 221; B 115 and 98; 1600 x 6400 in two parts, whose rests are more than half a round, 998 us whole, 948 so).
struct Cut {
    int32_t tile;
    int64_t slots;
    uint32_t rest, split;
    double us;
};
// What partial sums may take, in elements: slots leave at most two tiles each, pieces one.
constexpr int64_t kPartials = 512 * 2 * 128 * 128;

Cut group_cut(const OrthoLaunch& a, int kind) {
    Cut best = {64, 0, 0, 0, 0};
    double least = -1, bytes = 0;  // bytes: of the operands
    for (int i = 0; i < a.count; ++i) {
        const double x = (double)a.it[i].rp * a.it[i].cp, d = (double)std::min(a.it[i].rp, a.it[i].cp);
        bytes += 2.0 * a.parts * (kind == kGram ? x : kind == kPoly ? d * d : x + d * d);
    }
    const double rate = bytes < 8e6 ? 17e6 : bytes < 100e6 ? 7e6 : 4.4e6;  // bytes a us, from the L2s, the last-level cache and memory
    const int parts = 2 * a.parts;
    for (const int tile : {64, 128, 256}) {
        const int segs = mm_segments(tile, parts);
        int64_t tiles = 0, turns = 0;
        int32_t most = 0, same = 1;
        for (int i = 0; i < a.count; ++i) {
            const int64_t n = item_tiles(a.it[i], kind, tile);
            const int32_t t = item_turns(a.it[i], kind);
            if (i > 0 && t != most) same = 0;
            tiles += n;
            turns += n * t * segs;
            most = std::max(most, t);
        }
        const double mean = (double)turns / (double)tiles;  // turns of all segments
        // tiles of different lengths: the longest begin first
        const double whole = same ? mm_time(tile, tiles, most, parts) : std::max(mm_time(tile, 1, most, parts), mm_time(tile, tiles, (int64_t)std::ceil(mean / segs), parts));
        if (least < 0 || whole < least) least = whole, best = {tile, 0, 0, 0, whole};
        const int64_t round = 256 * mm_fit(tile, parts), rest = tiles % round;
        const double n = (double)most * segs;
        if (same && rest > 0)
            for (const int64_t rounds : {1, 2, 3}) {
                const int64_t split = std::min<int64_t>(rounds * round / rest, segs * most / (tile > 128 ? 8 : 4)), pieces = rest * split;
                if (split < 2) continue;  // a rest of more than half a round in one round
                if (pieces * tile * tile > kPartials) break;
                const double t = mm_time(tile, tiles - rest, most, parts) + (double)rounds * (mm_ends(tile, std::min(pieces, round), parts) + std::ceil(n / (double)split) * mm_turn(tile, std::min(pieces, round), parts)) +
                                 9 + (double)(pieces * tile * tile) * 4 / 4e6;
                if (t < least) least = t, best = {tile, 0, (uint32_t)rest, (uint32_t)split, t};
            }
        for (const int64_t slots : {16, 32, 64, 128, 256, 512}) {
            if (tile == 256 || slots > 256 * mm_fit(tile, parts) || turns < 4 * slots) break;
            const double turn = std::max(mm_turn(tile, slots, parts), (double)(slots * tile * 128 * (segs > 1 ? 2 : parts)) / rate), w = (double)turns / (double)slots,
                         pieces = std::min((double)(2 * slots), (double)(slots + tiles)),
                         t = 2 + w * turn + (w / mean + 1) * (mm_ends(tile, slots, parts) + 1) + 5 + pieces * tile * tile * 4 / 4e6;
            if (t < least) least = t, best = {tile, slots, 0, 0, t};
        }
    }
    return best;
}

template <int KIND>
hipError_t product(OrthoLaunch& a, hipStream_t st) {
    const Cut c = group_cut(a, KIND);
    a.slots = c.slots;
    a.rest = c.rest;
    a.split = c.split;
    a.begin[0] = 0;
    for (int i = 0; i < a.count; ++i)
        a.begin[i + 1] = a.begin[i] + item_tiles(a.it[i], KIND, c.tile) * (c.slots ? item_turns(a.it[i], KIND) * item_segments(c.tile, a.parts) : 1);
    if (c.tile == 64) return a.parts > 1 ? launch<64, KIND, 2>(a, st) : launch<64, KIND, 1>(a, st);
    return c.tile == 256 ? launch<256, KIND, 1>(a, st) : launch<128, KIND, 1>(a, st);
}

// Whether a group's steps are taken two at a time: three products of square matrices against X X^T and one with X, where the measured times say that this saves 25 us
// a pair (4096 x 11008 in one part: 3 x 98 us against 602; in two parts three matrices of 2048 x 5632, two of 2048 x 2048 and two small ones: 3 x 187
// against 931. 1001 x 1750 in two parts: 3 x 17 against 42; the ends of small products take longer than the times say).
bool in_pairs(const OrthoLaunch& a, const OrthoCoefs& k) {
    return k.pairs && k.steps > 1 && group_cut(a, kGram).us + group_cut(a, kNext).us > 3 * group_cut(a, kPoly).us + 25;
}

// Whether each tile of X takes b A + c A A for itself: one tile of it, and no more than a round of X's.
bool is_narrow(const OrthoItem& t) { return std::min(t.rp, t.cp) == 64 && std::max(t.rp, t.cp) <= 64 * 256; }
bool is_narrow(const OrthoLaunch& a) {
    for (int i = 0; i < a.count; ++i)
        if (!is_narrow(a.it[i])) return false;
    return true;
}
constexpr int32_t kSquares = 3;  // places for square matrices, and behind them the tiles' own

template <int KIND>
hipError_t narrow_product(OrthoLaunch& a, hipStream_t st) {
    a.slots = 0;
    a.rest = 0;
    uint32_t most = 0;
    for (int i = 0; i < a.count; ++i) {
        const int64_t n = item_tiles(a.it[i], KIND, 64);
        a.begin[i + 1] = a.begin[i] + n;
        most += (uint32_t)((n + 7) / 8);
    }
    a.whole = (uint32_t)a.begin[a.count];
    if (a.parts > 1)
        ortho_narrow_kernel<KIND, 2><<<8 * most, MmTile<64>::kThreads, 0, st>>>(a);
    else
        ortho_narrow_kernel<KIND, 1><<<8 * most, MmTile<64>::kThreads, 0, st>>>(a);
    return hipGetLastError();
}

// The steps of a group whose X0 lies in place 1; the last one's outputs go where LAST says.
template <int LAST>
hipError_t iterate(OrthoLaunch& a, const OrthoCoefs& k, hipStream_t st) {
    a.parts = k.parts;
    constexpr float kA = kAScale, kB = kBScale;
    const Square poly = {0, 0, 0, 0, 1, k.c * (kB / (kA * kA)), k.b * (kB / kA), 0};
    const Square pair[5] = {
        poly,                                                               // B, at 1
        {1, 0, 0, 0, 2, 1 / kB, k.a, 0},                                    // Y = a A + B A, at 2
        {2, 1, 2, 0, 0, 1 / kB, k.a, 0},                                    // A' = a Y + Y B, at 0
        {0, 0, 0, 0, 2, k.c * (kB / (kA * kA)), k.b * (kB / kA), 0},        // B', at 2
        {2, 1, 1, 2, 0, 1 / kB, k.a, k.a},                                  // D = a B + a B' + B' B, at 0
    };
    const bool narrow = is_narrow(a), pairs = !narrow && in_pairs(a, k);
    a.from = 1;
    a.first = 1;
    for (int i = 0; i < k.steps;) {
        const bool two = pairs && i + 1 < k.steps;
        hipError_t e = product<kGram>(a, st);
        if (narrow) {
            a.square = poly;
            a.square.out = a.by = kSquares;
            a.ca = k.a;
            ++i;
            if (e == hipSuccess) e = i < k.steps ? narrow_product<kNext>(a, st) : narrow_product<LAST>(a, st);
            if (e != hipSuccess) return e;
            a.from ^= 1;
            a.first = 0;
            continue;
        }
        for (int j = 0; j < (two ? 5 : 1) && e == hipSuccess; ++j) {
            a.square = two ? pair[j] : poly;
            e = product<kPoly>(a, st);
        }
        a.by = two ? 0 : 1;
        a.ca = two ? k.a * k.a : k.a;
        i += two ? 2 : 1;
        if (e == hipSuccess) e = i < k.steps ? product<kNext>(a, st) : product<LAST>(a, st);
        if (e != hipSuccess) return e;
        a.from ^= 1;
        a.first = 0;
    }
    return hipSuccess;
}

size_t up(size_t x) { return (x + 255) & ~size_t(255); }
int32_t padded(int64_t n) { return (int32_t)((n + 63) / 64 * 64); }

size_t first_bytes(const OrthoItem& t, int32_t parts, bool update) { return up((size_t)t.rp * t.cp * std::max(update ? 4 : 2, 2 * parts)); }

// Places of an item in the workspace from `at` on; returns the first byte behind.
char* place(OrthoItem& t, int64_t rows, int64_t cols, int32_t parts, bool update, char* at) {
    t.rows = (int32_t)rows;
    t.cols = (int32_t)cols;
    t.rp = padded(rows);
    t.cp = padded(cols);
    t.x[0] = reinterpret_cast<uint16_t*>(at);
    at += first_bytes(t, parts, update);
    t.x[1] = reinterpret_cast<uint16_t*>(at);
    at += up((size_t)t.rp * t.cp * 2 * parts);
    t.a = reinterpret_cast<uint16_t*>(at);
    const size_t d = (size_t)std::min(t.rp, t.cp);
    return at + up(d * d * 2 * parts * (kSquares + (is_narrow(t) ? (size_t)std::max(t.rp, t.cp) / 64 : 0)));
}

}  // namespace

size_t ortho_item_bytes(int64_t rows, int64_t cols, int32_t parts, bool update) {
    OrthoItem t = {};
    return (size_t)(place(t, rows, cols, parts, update, nullptr) - static_cast<char*>(nullptr));
}

int64_t ortho_sums(int64_t rows, int64_t cols) { return (rows * cols + kSquareUnit - 1) / kSquareUnit; }

int64_t ortho_turns(int64_t rows, int64_t cols, int32_t parts) {
    const int64_t r = padded(rows) / 64, c = padded(cols) / 64, d = std::min(r, c);
    return std::max(d * (d + 1) / 2 * std::max(r, c), r * c * d) * (parts > 1 ? 3 : 1);
}

// A slot has at least 4 turns and leaves at most two tiles of sums of 128 x 128 outputs at most, a piece has 4 of those and leaves one, or 8 of 256 x 256 outputs.
size_t ortho_part_bytes(int64_t turns) { return (size_t)std::min<int64_t>(kPartials, turns / 4 * 2 * 128 * 128) * 4; }

size_t ortho_part_bytes(int64_t rows, int64_t cols, int32_t parts) {
    OrthoLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.count = 1;
    a.parts = parts;
    place(a.it[0], rows, cols, parts, false, nullptr);
    size_t most = 0;
    for (const int kind : {kGram, kPoly, kNext}) {
        const Cut c = group_cut(a, kind);
        most = std::max(most, ((size_t)c.slots * 2 + (size_t)c.rest * c.split) * c.tile * c.tile * 4);
    }
    return most;
}

size_t ortho_head_bytes(int64_t sums) { return up(kOrthoGroup * sizeof(Norm)) + up((size_t)sums * 8); }

hipError_t launch_orthogonalize(int64_t rows, int64_t cols, const OrthoCoefs& k, int dtype, const void* x, int64_t ldx, int out_dtype, void* out, int64_t ldout,
                                void* ws, hipStream_t st) {
    char* const w = static_cast<char*>(ws);
    const int64_t units = ortho_sums(rows, cols);
    Norm* const norms = reinterpret_cast<Norm*>(w);
    double* const sums = reinterpret_cast<double*>(w + up(kOrthoGroup * sizeof(Norm)));
    char* at = w + ortho_head_bytes(units);
    OrthoLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.count = 1;
    a.norms = norms;
    a.part = reinterpret_cast<float*>(at);
    place(a.it[0], rows, cols, k.parts, false, at + ortho_part_bytes(rows, cols, k.parts));
    a.out = out;
    a.ldout = ldout;
    a.out_bf16 = out_dtype == AL_DTYPE_BF16;
    const uint32_t slabs = (uint32_t)std::min<int64_t>(units, kMostSums);
    PackList l;
    std::memset(&l, 0, sizeof(l));
    l.count = 1;
    l.t[0] = {x, ldx, a.it[0].x[1], a.it[0].rows, a.it[0].cols, a.it[0].rp, a.it[0].cp};
    l.begin[1] = (uint32_t)((int64_t)a.it[0].rp * a.it[0].cp / 2048);
    l.sums[1] = slabs;
    if (dtype == AL_DTYPE_BF16) {
        square_kernel<bf16><<<slabs, 256, 0, st>>>(static_cast<const bf16*>(x), ldx, rows, (int)cols, sums);
        pack_kernel<bf16><<<l.begin[1], 256, 0, st>>>(l, k.parts, k.eps, sums, norms);
    } else {
        square_kernel<float><<<slabs, 256, 0, st>>>(static_cast<const float*>(x), ldx, rows, (int)cols, sums);
        pack_kernel<float><<<l.begin[1], 256, 0, st>>>(l, k.parts, k.eps, sums, norms);
    }
    return iterate<kOut>(a, k, st);
}

hipError_t launch_muon(const MuonItem* items, int count, const OrthoCoefs& k, const MuonArgs& m, void* ws, hipStream_t st) {
    char* const w = static_cast<char*>(ws);
    int64_t units = 0, turns = 0;
    for (int i = 0; i < count; ++i) units += ortho_sums(items[i].rows, items[i].cols), turns += ortho_turns(items[i].rows, items[i].cols, k.parts);
    Norm* const norms = reinterpret_cast<Norm*>(w);
    double* const sums = reinterpret_cast<double*>(w + up(kOrthoGroup * sizeof(Norm)));
    char* at = w + ortho_head_bytes(units);
    OrthoLaunch a;
    MomentumList l;
    PackList q;
    std::memset(&a, 0, sizeof(a));
    std::memset(&l, 0, sizeof(l));
    std::memset(&q, 0, sizeof(q));
    a.count = l.count = q.count = count;
    a.norms = norms;
    a.part = reinterpret_cast<float*>(at);
    a.decay = m.decay;
    at += ortho_part_bytes(turns);
    for (int i = 0; i < count; ++i) {
        const MuonItem& s = items[i];
        OrthoItem& t = a.it[i];
        at = place(t, s.rows, s.cols, k.parts, true, at);
        t.p = s.p;
        t.step = s.step;
        float* const u = reinterpret_cast<float*>(t.x[0]);
        l.t[i] = {s.g, s.m, s.meta, u, s.rows * s.cols};
        l.begin[i + 1] = l.begin[i] + (uint32_t)ortho_sums(s.rows, s.cols);
        q.t[i] = {u, s.cols, t.x[1], t.rows, t.cols, t.rp, t.cp};
        q.begin[i + 1] = q.begin[i] + (uint32_t)((int64_t)t.rp * t.cp / 2048);
        q.sums[i + 1] = l.begin[i + 1];
    }
    const hipError_t e = launch_momentum(m, l, sums, st);
    if (e != hipSuccess) return e;
    for (int i = 0; i < count; ++i)
        if (q.sums[i + 1] - q.sums[i] > kMostSums) {
            norm_kernel<<<(uint32_t)count, 256, 0, st>>>(q, k.eps, sums, norms);
            break;
        }
    pack_kernel<float><<<q.begin[count], 256, 0, st>>>(q, k.parts, k.eps, sums, norms);
    return iterate<kStep>(a, k, st);
}

}  // namespace al
