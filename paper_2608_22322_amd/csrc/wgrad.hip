// Weight gradient of a linear layer from its input's E8 code, on the matrix
// cores: dw[n][k] = sum over tokens t of dy[t][n] xhat[t][k].
//
// Both factors are bf16 numbers (a code is 7 bits and a sign times a power of two; an
// fp32 dy is the sum of three bf16 numbers, taken in three turns, but for bits below bf16's
// smallest number, 2^-133), so every product is exact and the sums are the matrix cores' fp32 ones. A workgroup
// decodes each code once, on its way to LDS (2.5 instructions a value: convert a
// byte, multiply, pack; the fragments' readers would do it twice or four times).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "act_device.hpp"

namespace al {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) uint16_t* lds_u16;

// Both tiles lie in LDS as they do in memory, a row per token. A transposing read gives lane l of
// a wavefront the 4 tokens 4 (l / 16) + 0..3 of column l % 16: two of them make the 8-token fragment of
// a 16 x 16 x 32 product (which token comes at which place does not matter, as both factors
// agree). Half a wavefront reads one 32-byte unit of each of 8 rows at once; the units of a row are exchanged so that
// these lie in different banks.
constexpr int kTurn = 32;  // tokens a turn
constexpr int kBig = 256, kMid = 128, kEdge = 64;  // tile widths
constexpr int64_t kBeside = 16384;  // most tokens at which a split product's launch also takes the sums of dy

__device__ __forceinline__ int edge_at(int t, int c) { return t * kEdge + ((((c >> 4) ^ ((t >> 1) & 3)) << 4) | (c & 15)); }

// The bf16 part `which` (0, 1, 2) of fp32 values: x = x0 + x1 + x2 down to bits of 2^-133, by truncation; infinities and NaN
// are in part 0 alone.
__device__ __forceinline__ uint32_t split_part(uint32_t x, int which) {
    const bool fin = (x & 0x7f800000u) != 0x7f800000u;
    if (!fin) return which == 0 ? (x & 0x007fffffu ? 0x7fc0u : x >> 16) : 0u;
    const uint32_t h = x & 0xffff0000u;
    if (which == 0) return h >> 16;
    const float r = bits_f(x) - bits_f(h);
    const uint32_t m = f_bits(r) & 0xffff0000u;
    if (which == 1) return m >> 16;
    return f_bits(r - bits_f(m)) >> 16;
}

template <typename T>
__device__ __forceinline__ u32x4 as_bf16(const Chunk<T>& k, int which);
template <>
__device__ __forceinline__ u32x4 as_bf16<bf16>(const Chunk<bf16>& k, int) {
    return k.q;
}
template <>
__device__ __forceinline__ u32x4 as_bf16<float>(const Chunk<float>& k, int which) {
    u32x4 q;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        q[j] = split_part(k.a[2 * j], which) | split_part(k.a[2 * j + 1], which) << 16;
        q[2 + j] = split_part(k.b[2 * j], which) | split_part(k.b[2 * j + 1], which) << 16;
    }
    return q;
}

__device__ __forceinline__ bf16x8 tile_fragment(const uint16_t* tile, int at0, int at1) {
    union {
        s16x4 h[2];
        bf16x8 f;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds_u16)(uint16_t*)(tile + at0));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds_u16)(uint16_t*)(tile + at1));
    return u.f;
}

// Eight codes as bf16 numbers.
__device__ __forceinline__ u32x4 decode_bf16(u32x2 codes, uint32_t e) {
    float v[8];
    e8_decode(codes, e, v);
    u32x4 q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = __builtin_amdgcn_perm(f_bits(v[2 * j + 1]), f_bits(v[2 * j]), 0x07060302u);
    return q;
}

__device__ __forceinline__ float grad_at(const bf16* p, int64_t i) { return to_f(p[i]); }
__device__ __forceinline__ float grad_at(const float* p, int64_t i) { return p[i]; }

// One finished sum: scale, shift (t(): the sum of dy's column n), base, and the only rounding.
template <typename O, typename F>
__device__ __forceinline__ void finish(const Wgrad& a, int64_t n, int k, float v, const F& t) {
    const int64_t i = n * a.s.cols + k;
    if (a.gamma) v *= a.gamma[k];
    if (a.beta) v += a.beta[k] * t();
    if (a.base) v += grad_at(static_cast<const O*>(a.base), i);
    put(static_cast<O*>(a.dw) + i, v);
}

// Four finished sums of consecutive columns k.. of row n (in: how many of them lie inside).
template <typename O, typename F>
__device__ __forceinline__ void finish4(const Wgrad& a, int64_t n, int k, int in, f32x4 v, const F& t) {
    if (in < 4) {
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < in) finish<O>(a, n, k + r, v[r], t);
        return;
    }
    typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
    const int64_t i = n * a.s.cols + k;
    if (a.gamma) v *= *reinterpret_cast<const f32x4_a4*>(a.gamma + k);
    if (a.beta) {
        const f32x4 b = *reinterpret_cast<const f32x4_a4*>(a.beta + k);
        const float s = t();
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += b[r] * s;
    }
    if constexpr (sizeof(O) == 4) {
        if (a.base) v += *reinterpret_cast<const f32x4_a4*>(static_cast<const float*>(a.base) + i);
        *reinterpret_cast<f32x4_a4*>(static_cast<float*>(a.dw) + i) = v;
    } else {
        typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
        if (a.base) {
            const u32x2 b = *reinterpret_cast<const u32x2_a2*>(static_cast<const bf16*>(a.base) + i);
#pragma unroll
            for (int r = 0; r < 2; ++r) v[2 * r] += bits_f(b[r] << 16), v[2 * r + 1] += bits_f(b[r] & 0xffff0000u);
        }
        *reinterpret_cast<u32x2_a2*>(static_cast<bf16*>(a.dw) + i) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
}

// The shape of the products, M x M. 16 x 16 x 32 takes more cycles than 32 x 32 x 16 and keeps a higher clock (8192 tokens and
// features: 1.85M cycles at 2.13 GHz against 1.74M at 1.92 GHz), so bf16 dy takes it; fp32 dy, whose staging needs the
// registers that fewer fragments in flight leave, takes 32 x 32 x 16 (4096^3: 842 and 414 us).
template <int M>
struct Product;
template <>
struct Product<16> {
    typedef f32x4 acc_t;
    static constexpr int kTokens = 32, kQuads = 1;
    // unit u (32 bytes) of row t lies at u ^ t % 16: half a wavefront reads one unit of 8 rows, all 64 banks
    static __device__ __forceinline__ int swizzle(int t) { return t & 15; }
    // a transposing read gives lanes 16 g .. 16 g + 15 columns 0..15 of tokens 4 g .. 4 g + 3, a second one 16 tokens on
    static __device__ __forceinline__ int token(int lane) { return 4 * (lane >> 4) + ((lane >> 2) & 3); }
    static __device__ __forceinline__ int column(int lane) { return 4 * (lane & 3); }
    // columns (k) of a lane's sums: 4 (l / 16) + 0..3
    static __device__ __forceinline__ int quad(int lane, int) { return 4 * (lane >> 4); }
    static __device__ __forceinline__ acc_t mul(bf16x8 x, bf16x8 y, acc_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    }
};
template <>
struct Product<32> {
    typedef f32x16 acc_t;
    static constexpr int kTokens = 16, kQuads = 4;
    // u ^ 2 (t % 8): half a wavefront reads two units of 4 rows
    static __device__ __forceinline__ int swizzle(int t) { return (t & 7) << 1; }
    // lanes 16 g ..: columns 16 (g % 2) .. of tokens 4 (g / 2) ..; a second one 8 tokens on
    static __device__ __forceinline__ int token(int lane) { return 4 * (lane >> 5) + ((lane >> 2) & 3); }
    static __device__ __forceinline__ int column(int lane) { return (lane & 16) + 4 * (lane & 3); }
    static __device__ __forceinline__ int quad(int lane, int q) { return 8 * q + 4 * (lane >> 5); }
    static __device__ __forceinline__ acc_t mul(bf16x8 x, bf16x8 y, acc_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
    }
};

// A B x B tile's outputs: wavefront w holds rows WN (w / (B / WK)) .., columns WK (w % (B / WK)) .. as FN x FK blocks of M x M, a lane
// four consecutive columns of one row in each of a block's quads.
template <int B, int M>
struct Tile {
    static constexpr int WN = B / 2, WK = B == kEdge ? 32 : 64, FN = WN / M, FK = WK / M, kQuads = Product<M>::kQuads,
                         kWaves = (B / WN) * (B / WK), kSlots = FN * FK * kQuads;
    int n_first, n0, k_first, k0;  // what the tile is answerable for begins at n_first, k_first; its first output is n0, k0
    __device__ __forceinline__ Tile(const Wgrad& a, int n, int k) {
        n_first = n0 = n * B;
        k_first = k0 = k * B;
        if (B != kEdge) n0 = std::min(n0, (int)a.out - B), k0 = std::min(k0, a.s.pitch - B);
    }
    static __device__ __forceinline__ int wave_n(int w) { return w / (B / WK) * WN; }
    static __device__ __forceinline__ int wave_k(int w) { return w % (B / WK) * WK; }
    // row, first column and number of columns of a lane's quad (0: none of this tile's)
    __device__ __forceinline__ int quad(const Wgrad& a, int w, int i, int j, int q, int lane, int& n, int& k) const {
        n = n0 + wave_n(w) + M * i + (lane & (M - 1));
        k = k0 + wave_k(w) + M * j + Product<M>::quad(lane, q);
        return n < n_first || n >= a.out || k < k_first ? 0 : std::min(4, a.s.cols - k);
    }
};

// The sums of a workgroup's tile: finished, or, where the tokens are split, as partial products in the order in which the lanes hold
// them (whole lines; the outputs' own order takes 16-byte pieces and 3 times as long): [split][tile][wavefront][slot][lane].
template <typename O, int B, int M, typename ACC>
__device__ __forceinline__ void write_tile(const Wgrad& a, const Tile<B, M>& t, int64_t tile, int64_t tiles, int split, int w, int lane,
                                           const ACC& acc) {
    typedef Tile<B, M> G;
    f32x4* const part = reinterpret_cast<f32x4*>(a.part) + ((split * tiles + tile) * G::kWaves + w) * G::kSlots * 64 + lane;
    // (One row of blocks at a time: with all their loads in flight at once the sums would not stay in registers.)
#pragma unroll
    for (int i = 0; i < G::FN; ++i) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < G::FK; ++j) {
#pragma unroll
            for (int q = 0; q < G::kQuads; ++q) {
                f32x4 v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r];
                if (a.splits > 1) {
                    part[((i * G::FK + j) * G::kQuads + q) * 64] = v;
                } else {
                    int n, k;
                    const int in = t.quad(a, w, i, j, q, lane, n, k);
                    if (in > 0) finish4<O>(a, n, k, in, v, [&] { return a.bsum[n]; });
                }
            }
        }
    }
}

// Column sums of dy over one of bparts slabs of tokens, 512 columns (at = slab + bparts * block of columns): 8 columns a lane, W
// wavefronts, 8 rows of each in flight; buf: (W - 1) * 512 floats of LDS.
template <typename T, int W>
__device__ __forceinline__ void sum_dy(const Wgrad& a, uint32_t at, float* part, float* buf) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, slab = (int)(at % (uint32_t)a.bparts);
    const int c = (int)(at / (uint32_t)a.bparts * 64 + lane) * 8, out = (int)a.out;
    float s[8] = {};
    if (c < out) {
        const int64_t r0 = a.s.rows * slab / a.bparts, r1 = a.s.rows * (slab + 1) / a.bparts;
        for (int64_t r = r0 + w; r < r1; r += 8 * W) {
            Chunk<T> k[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                k[i].zero();
                if (r + i * W < r1) load_chunk(k[i], static_cast<const T*>(a.dy.p) + (r + i * W) * a.dy.ld, c, out);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v[8];
                k[i].get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += v[j];
            }
        }
    }
    if (w > 0)
#pragma unroll
        for (int j = 0; j < 8; ++j) buf[(w - 1) * 512 + j * 64 + lane] = s[j];
    __syncthreads();
    if (w > 0 || c >= out) return;
    for (int i = 0; i < W - 1; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += buf[i * 512 + j * 64 + lane];
    store_chunk(part + a.out * slab, c, out, s);
}

// The splits' partial products, added in order, 8 splits' loads in flight; the slabs' sums of dy likewise, which the lanes that hold
// column 0 write as the bias gradient.
template <typename O, int B, int M>
__global__ __launch_bounds__(256) void wgrad_join_kernel(Wgrad a, FastDiv kt, uint32_t tiles) {
    typedef Tile<B, M> G;
    constexpr uint32_t kBlocks = B * B / 1024;  // workgroups a tile
    const uint32_t id = xcd_block(blockIdx.x, gridDim.x), tile = id / kBlocks, at = id % kBlocks * 256 + threadIdx.x, lane = at & 63, slot = at >> 6;
    const int64_t size = (int64_t)tiles * (B * B / 4);
    const f32x4* p = reinterpret_cast<const f32x4*>(a.part) + (int64_t)tile * (B * B / 4) + at;
    f32x4 v = {};
    int s = 0;
    for (; s + 8 <= a.splits; s += 8, p += 8 * size) {
        f32x4 t[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) t[r] = p[r * size];
#pragma unroll
        for (int r = 0; r < 8; ++r) v += t[r];
    }
    for (; s < a.splits; ++s, p += size) v += *p;
    const int w = slot / G::kSlots, e = slot % G::kSlots, tn = (int)quotient(tile, kt);
    int n, k;
    const int in = G(a, tn, (int)(tile - (uint32_t)tn * kt.d))
                       .quad(a, w, e / (G::FK * G::kQuads), e / G::kQuads % G::FK, e % G::kQuads, (int)lane, n, k);
    if (in <= 0) return;
    float t = 0.0f;
    if (a.beta && !a.sums) t = a.bsum[n];
    if (a.sums && (a.beta || (a.dbias && k == 0))) {
        for (int i = 0; i < a.bparts; i += 8) {  // a multiple of 8 here
            float u[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) u[r] = a.bsum[(int64_t)(i + r) * a.out + n];
#pragma unroll
            for (int r = 0; r < 8; ++r) t += u[r];
        }
        if (a.dbias && k == 0) put(static_cast<O*>(a.dbias) + n, t);
    }
    finish4<O>(a, n, k, in, v, [&] { return t; });
}

// 64 x 64 outputs, 4 wavefronts of 32 x 32, any size and alignment. A turn is short here, so the loads of AHEAD of them are
// in flight. Loads are never masked: rows past the last are the last one's and columns past a side's end its last ones, of which
// the former are cleared on the way to LDS and the latter make sums that are not written.
template <typename T, typename O, bool SUMS>
__global__ __launch_bounds__(256) void wgrad_edge_kernel(Wgrad a) {
    __shared__ __attribute__((aligned(16))) uint16_t dy_s[2][kTurn * kEdge], x_s[2][kTurn * kEdge];
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, AHEAD = 4;
    int split = (int)blockIdx.z;
    if (SUMS) {  // the first layers of the grid take the sums of dy (a kernel of its own: 0.5 of 9 us where there are none)
        split -= (int)gridDim.z - a.splits;
        if (split < 0) {
            const uint32_t at = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
            if (at < a.sums) sum_dy<T, 4>(a, at, a.bsum, reinterpret_cast<float*>(dy_s));
            return;
        }
    }
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t n0 = (int64_t)blockIdx.y * kEdge;
    const int k0 = blockIdx.x * kEdge;
    // this split's tokens
    const int64_t steps = (a.s.rows + kTurn - 1) / kTurn;
    const int64_t s0 = steps * split / a.splits, s1 = steps * (split + 1) / a.splits;

    const int cc = (tid & 7) * 8, t0 = tid >> 3;  // this thread's columns and token of a step
    const int out = (int)a.out, c = (int)n0 + cc, from = std::max(0, std::min(c, out - 8)), shift = std::min(c - from, 8);
    const int xc = std::min(k0 + cc, a.s.pitch - 8);
    const T* const dyp = static_cast<const T*>(a.dy.p) + from;
    Chunk<T> dy[AHEAD];
    u32x2 xq[AHEAD];
    uint32_t xe[AHEAD];
    const auto load = [&](int i, int64_t step) __attribute__((always_inline)) {
        const int64_t t = std::min(step * kTurn + t0, a.s.rows - 1);
        if (out >= 8)
            dy[i].load(dyp + t * a.dy.ld);
        else
            dy[i].load(dyp + t * a.dy.ld, out);
        xq[i] = *reinterpret_cast<const u32x2*>(a.c.p + t * a.s.pitch + xc);
        xe[i] = a.c.e[t * a.s.nb + (xc >> (3 + a.s.lb))];
    };
    const auto fragment = [&](const uint16_t* tile, int c0) __attribute__((always_inline)) {
        const int t = 4 * (lane >> 4) + ((lane >> 2) & 3), f = c0 + 4 * (lane & 3);
        return tile_fragment(tile, edge_at(t, f), edge_at(t + 16, f));
    };
    const int wn = Tile<kEdge, 16>::wave_n(w), wk = Tile<kEdge, 16>::wave_k(w);
    f32x4 acc[2][2] = {};
    int b = 0;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (s0 + i < s1) load(i, s0 + i);
    for (int64_t s = s0; s < s1; s += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (s + i >= s1) break;
            if (shift > 0 && out >= 8) dy[i].drop(shift & 7);
            if ((s + i) * kTurn + t0 >= a.s.rows) {
                dy[i].zero();
                xq[i] = 0u;
                xe[i] = 0u;
            }
#pragma unroll
            for (int part = 0; part < PARTS; ++part, b ^= 1) {
                *reinterpret_cast<u32x4*>(&dy_s[b][edge_at(t0, cc)]) = as_bf16<T>(dy[i], part);
                *reinterpret_cast<u32x4*>(&x_s[b][edge_at(t0, cc)]) = decode_bf16(xq[i], xe[i]);
                if (part == PARTS - 1 && s + i + AHEAD < s1) load(i, s + i + AHEAD);
                __syncthreads();
                bf16x8 fx[2], fy[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    fx[r] = fragment(x_s[b], wk + 16 * r);
                    fy[r] = fragment(dy_s[b], wn + 16 * r);
                }
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[j], fy[r], acc[r][j], 0, 0, 0);
            }
        }
    }
    write_tile<O>(a, Tile<kEdge, 16>(a, blockIdx.y, blockIdx.x), (int64_t)blockIdx.y * gridDim.x + blockIdx.x, (int64_t)gridDim.x * gridDim.y,
                  split, w, lane, acc);
}

template <int B, int M>
__device__ __forceinline__ int tile_at(int t, int c) {
    return t * B + ((((c >> 4) ^ (Product<M>::swizzle(t) & (B / 16 - 1))) << 4) | (c & 15));
}

// Workgroup -> tile. An XCD takes a contiguous share of the tiles, in bands of 8 along n: the 32 that it works on at a time
// are 8 x 4, so each of their rows and columns of tiles is read from memory once and by the others from the XCD's L2.
struct TileId {
    int n, k, split;
};
constexpr uint32_t kBand = 8;
template <int B>
__device__ __forceinline__ TileId tile_id(const Wgrad& a) {
    const uint32_t nt = (uint32_t)((a.out + B - 1) / B), kt = (uint32_t)((a.s.cols + B - 1) / B);
    const uint32_t id = xcd_block(blockIdx.x - a.sums, gridDim.x - a.sums), split = id / (nt * kt), r = id - split * (nt * kt), band = r / (kBand * kt),
                   rows = min(kBand, nt - band * kBand), q = r - band * kBand * kt, k = q / rows;
    return {(int)(band * kBand + q - k * rows), (int)k, (int)split};
}

// B x B outputs, for out_features and in_features of at least B: the last tile of a side is moved back to end with it, so that no
// load needs a bounds check, and leaves what the tile before it has written. B = 256: 8 wavefronts of 128 x 64 (2 along n, 4 along
// k), one workgroup per compute unit; B = 128: 4 wavefronts of 64 x 64, up to three.
//
// 8192^3 bf16: 905 us, 1.21 PFLOP/s (a library product of bf16 matrices in these orders: 1.15; 1.27 in its best order). The matrix
// units are busy 57% of the cycles at 2.13 GHz; 100% of them at the nominal 2.4 would be 2.5 PFLOP/s. Of the rest a part is
// power: the same products in fewer cycles (32 x 32 x 16, 60%) ran at 1.92 GHz and took longer. What got it there, us for 8192 tokens,
// 11008 x 4096: 128 x 128 tiles 1045; 256 x 256 with the next tiles staged beside the products 819; offsets from scalar bases and
// no branches in the turns 780; fragments two ahead and the decoding between matrix instructions 683; bands per XCD 670.
template <typename T, typename O, int B>
__global__ __launch_bounds__(2 * B, B == kBig ? 2 : 3) void wgrad_tile_kernel(Wgrad a) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, BT = kTurn, C = BT / 16;
    constexpr int M = PARTS == 1 ? 16 : 32, FN = Tile<B, M>::FN, FK = Tile<B, M>::FK, H = BT / Product<M>::kTokens;
    __shared__ __attribute__((aligned(16))) uint16_t dy_s[2][BT * B], x_s[2][BT * B];
    if (blockIdx.x < a.sums) {  // sums of dy, where these are wanted and the tokens are split
        sum_dy<T, B / 32>(a, blockIdx.x, a.bsum, reinterpret_cast<float*>(dy_s));
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const TileId tile = tile_id<B>(a);
    typedef Tile<B, PARTS == 1 ? 16 : 32> G;
    const G t(a, tile.n, tile.k);
    const int n0 = t.n0, k0 = t.k0;
    const int64_t steps = (a.s.rows + BT - 1) / BT;
    const int64_t s0 = steps * tile.split / a.splits, s1 = steps * (tile.split + 1) / a.splits;

    // this thread stages columns 8 (tid % (B / 8)) .. + 7 of tokens tid / (B / 8) + 16 i: 32-bit offsets from a step's
    // first token
    const int cc = tid % (B / 8) * 8, t0 = tid / (B / 8);
    uint32_t od[C], ox[C], oe[C];
    const auto offsets = [&](int64_t step) __attribute__((always_inline)) {
        const int last = (int)std::min<int64_t>(a.s.rows - 1 - step * BT, BT - 1);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const uint32_t row = (uint32_t)std::min(t0 + 16 * i, last);
            od[i] = (row * (uint32_t)a.dy.ld + (uint32_t)cc) * (uint32_t)sizeof(T);
            ox[i] = row * (uint32_t)a.s.pitch + (uint32_t)cc;
            oe[i] = row * (uint32_t)a.s.nb + ((uint32_t)(k0 + cc) >> (3 + a.s.lb));
        }
    };
    Chunk<T> dy[C];
    u32x2 xq[C];
    uint32_t xe[C];
    const auto load = [&](int64_t step, bool whole) __attribute__((always_inline)) {
        const char* const dyp = reinterpret_cast<const char*>(static_cast<const T*>(a.dy.p) + step * BT * a.dy.ld + n0);
        const char* const xp = reinterpret_cast<const char*>(a.c.p) + step * BT * a.s.pitch + k0;
        const uint8_t* const ep = a.c.e + step * BT * a.s.nb;
        if (!whole && (step + 1) * BT > a.s.rows) offsets(step);  // the last step may be short
#pragma unroll
        for (int i = 0; i < C; ++i) {
            dy[i].load(reinterpret_cast<const T*>(dyp + od[i]));
            xq[i] = *reinterpret_cast<const u32x2*>(xp + ox[i]);
            xe[i] = ep[oe[i]];
        }
    };
    // rows past the split's last token add nothing
    const int64_t rows_end = std::min<int64_t>(a.s.rows, s1 * BT);
    const auto clip = [&](int64_t step) __attribute__((always_inline)) {
        if ((step + 1) * BT <= rows_end) return;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if (step * BT + t0 + 16 * i < rows_end) continue;
            dy[i].zero();
            xq[i] = 0u;
            xe[i] = 0u;
        }
    };
    const auto stage_dy = [&](uint16_t* tile, int part) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C; ++i) *reinterpret_cast<u32x4*>(&tile[tile_at<B, M>(t0 + 16 * i, cc)]) = as_bf16<T>(dy[i], part);
    };
    const auto stage_x = [&](uint16_t* tile) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            *reinterpret_cast<u32x4*>(&tile[tile_at<B, M>(t0 + 16 * i, cc)]) = decode_bf16(xq[i], xe[i]);
        }
    };

    const int wn = G::wave_n(w), wk = G::wave_k(w), ft = Product<M>::token(lane), fc = Product<M>::column(lane);
    int ay[FN][2], ax[FK][2];  // a fragment's two reads
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int i = 0; i < FN; ++i) ay[i][r] = tile_at<B, M>(ft + r * Product<M>::kTokens / 2, wn + M * i + fc);
#pragma unroll
        for (int j = 0; j < FK; ++j) ax[j][r] = tile_at<B, M>(ft + r * Product<M>::kTokens / 2, wk + M * j + fc);
    }
    typename Product<M>::acc_t acc[FN][FK] = {};
    const auto multiply = [&](const uint16_t* ty, const uint16_t* tx) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const int at = h * Product<M>::kTokens * B;
            bf16x8 fx[FK];
#pragma unroll
            for (int j = 0; j < FK; ++j) fx[j] = tile_fragment(tx + at, ax[j][0], ax[j][1]);
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const bf16x8 fy = tile_fragment(ty + at, ay[i][0], ay[i][1]);
#pragma unroll
                for (int j = 0; j < FK; ++j) acc[i][j] = Product<M>::mul(fx[j], fy, acc[i][j]);
            }
        }
    };
    if (s0 < s1) {
        offsets(s0);
        load(s0, false);
        clip(s0);
        stage_dy(dy_s[0], 0);
        stage_x(x_s[0]);
        if (PARTS == 1 && s0 + 1 < s1) load(s0 + 1, false);
    }
    __syncthreads();
    // One turn: this turn's products, and beside them the next turn's tiles into the other buffers and the loads after
    // those. WHOLE: every step that the turn looks at is 32 tokens of this split.
    const auto turn = [&](int64_t s, int part, int bd, int bx, auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        multiply(dy_s[bd], x_s[bx]);
        if (part + 1 < PARTS) {
            stage_dy(dy_s[bd ^ 1], part + 1);
            if (part + 1 == PARTS - 1 && (WHOLE || s + 1 < s1)) load(s + 1, WHOLE);
        } else {
            if (!WHOLE) clip(s + 1);
            stage_dy(dy_s[bd ^ 1], 0);
            stage_x(x_s[bx ^ 1]);
            if (PARTS == 1 && (WHOLE || s + 2 < s1)) load(s + 2, WHOLE);
        }
        if constexpr (WHOLE && M == 16) {
            // the matrix instructions with fragments two ahead, the decoding and the LDS writes between them, then the loads
            __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
            for (int i = 0; i < FN; ++i) {
#pragma unroll
                for (int j = 0; j < FK; ++j) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (j < 2 && i < FN - 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    if (i >= FN / 2) __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
                    if (i >= FN / 2 && j % 2 == 1 && (B != kBig || j == 3)) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                }
            }
            __builtin_amdgcn_sched_group_barrier(0x020, 6, 0);
        }
        __syncthreads();
    };
    const auto trip = [&](int64_t s, auto whole) __attribute__((always_inline)) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) turn(s, part, part & 1, 0, whole);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) turn(s + 1, part, (PARTS + part) & 1, 1, whole);
    };
    // two turns a trip, so that the buffers' addresses are constants; the second of a last odd one multiplies zeros
    const int64_t whole_end = std::min<int64_t>(s1, a.s.rows / BT);
    int64_t s = s0;
    for (; s + 3 < whole_end; s += 2) trip(s, std::true_type{});
    for (; s < s1; s += 2) trip(s, std::false_type{});
    const int64_t kt = (a.s.cols + B - 1) / B;
    write_tile<O>(a, t, tile.n * kt + tile.k, kt * ((a.out + B - 1) / B), tile.split, w, lane, acc);
}

template <typename T>
__global__ __launch_bounds__(256) void dy_sum_kernel(Wgrad a) {
    __shared__ float buf[3 * 512];
    sum_dy<T, 4>(a, blockIdx.x, a.bsum + a.out, buf);  // behind the whole sums
}

template <typename T, typename O, int B>
hipError_t launch_tile(const Wgrad& a, hipStream_t st) {
    const uint32_t kt = (uint32_t)((a.s.cols + B - 1) / B), tiles = kt * (uint32_t)((a.out + B - 1) / B);
    wgrad_tile_kernel<T, O, B><<<a.sums + tiles * (uint32_t)a.splits, 2 * B, 0, st>>>(a);
    if (a.splits > 1)
        wgrad_join_kernel<O, B, sizeof(T) == 2 ? 16 : 32><<<tiles * (B * B / 1024), 256, 0, st>>>(a, fast_div(kt), tiles);
    return hipGetLastError();
}

template <typename T, typename O>
hipError_t run(Wgrad a, hipStream_t st) {
    const uint32_t sums = a.bsum ? (uint32_t)((a.out + 511) / 512) * (uint32_t)a.bparts : 0u;
    if (a.bsum && !a.beside) {
        dy_sum_kernel<T><<<sums, 256, 0, st>>>(a);
        const FoldOut out = {a.dbias, a.bsum};
        const hipError_t e = launch_fold(sizeof(O) == 2 ? AL_DTYPE_BF16 : AL_DTYPE_F32, a.bsum + a.out, a.bparts, a.out, &out, 1, st);
        if (e != hipSuccess) return e;
    }
    a.sums = a.beside ? sums : 0u;
    if (a.s.cols == 0) return hipSuccess;
    // a plan's partial products have the layout of its tile; the large tiles' 32-bit offsets span 32 rows
    if (a.tile != kEdge && a.dy.ld < (1 << 25) && a.s.pitch < (1 << 26))
        return a.tile == kBig ? launch_tile<T, O, kBig>(a, st) : launch_tile<T, O, kMid>(a, st);
    dim3 n((uint32_t)((a.s.cols + kEdge - 1) / kEdge), (uint32_t)((a.out + kEdge - 1) / kEdge), (uint32_t)a.splits);
    const uint32_t tiles = n.x * n.y;
    n.z += (a.sums + tiles - 1) / tiles;
    if (a.sums) wgrad_edge_kernel<T, O, true><<<n, 256, 0, st>>>(a);
    else wgrad_edge_kernel<T, O, false><<<n, 256, 0, st>>>(a);
    if (a.splits > 1) {
        wgrad_join_kernel<O, kEdge, 16><<<tiles * (kEdge * kEdge / 1024), 256, 0, st>>>(a, fast_div(n.x), tiles);
    }
    return hipGetLastError();
}

}  // namespace

// The tile and the splits over the tokens that a measured model of the time finds shortest (us, one MI355X, fitted to 52 cases
// of both types, 1 to 16384 tokens and 64 x 64 to 11008 x 4096 outputs, each at every tile and up to 13 splits; its choices took 2%
// longer on average than each case's best, 16% at most):
//   a turn of a workgroup alone on its compute unit takes `alone`, of as many as fit beside each other `each` per workgroup;
//   starting and ending take as long as `ends` turns; fp32 dy takes 3 turns for one, each 10% longer; joining takes a launch
//   and the partial products' way out and back.
// Measured, the choice first: 8192 tokens, 11008 x 4096: 256-wide 651, 128-wide 836; 2048 x 2048: 256-wide 4 splits 78, 128-wide 3 splits 93;
// 1024 x 1024: 128-wide 8 splits 35, 256-wide 12 splits 38; 6001 tokens, 256 x 2048: 64-wide 6 splits 24.2 (8 splits 23.7), 128-wide 16 splits
// 25.4; 512 tokens, 1024 x 1024: 64-wide 8.6, 128-wide 13, 64-wide 2 splits 13.
WgradPlan wgrad_plan(int dtype, int64_t tokens, int64_t out, int64_t in) {
    static constexpr struct {
        int tile, fit, ends;
        double alone, each;
    } kinds[] = {{kEdge, 6, 1, 0.37, 0.13}, {kMid, 3, 2, 0.44, 0.28}, {kBig, 1, 6, 0.8, 0.8}};
    static constexpr int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
    const int64_t steps = std::max<int64_t>(1, (tokens + kTurn - 1) / kTurn);
    WgradPlan p;
    double best = 0;
    for (const auto& k : kinds) {
        if (k.tile != kEdge && std::min(out, in) < k.tile) continue;
        const int64_t n = std::max<int64_t>(1, ((out + k.tile - 1) / k.tile) * ((in + k.tile - 1) / k.tile));
        for (const int s : counts) {
            if (s > 1 && (2 * s > steps || n * s > 2048 || in == 0)) break;
            const double load = (double)(n * s) / 256, whole = std::ceil(load),
                         turns = (double)((steps + s - 1) / s) * (dtype == AL_DTYPE_BF16 ? 1 : 3.3) + k.ends,
                         turn = k.fit == 1 ? k.each * whole : load > k.fit ? k.each * load : std::max(k.alone, k.each * whole),
                         t = turns * turn + (s > 1 ? 2 + 0.02 * s + 0.34e-6 * 4 * s * (double)out * (double)in : 0);
            if (best == 0 || t < best) best = t, p.tile = k.tile, p.splits = s, p.part_bytes = s > 1 ? (size_t)(s * n) * k.tile * k.tile * 4 : 0;
        }
    }
    // Sums of dy: split products of at most kBeside tokens take them along, in few slabs, as each joining lane adds these up (two
    // launches less; bf16 with dbias: 512 x 256 x 256 16.1 -> 10.9 us, 6001 x 256 x 2048 31.7 -> 26.6, 16384 x 256 x 256 23.2 -> 19.1).
    // With more tokens a workgroup's slab takes longer than the product does (65536 x 256 x 256: 41 -> 69 us).
    p.beside = p.splits > 1 && tokens <= kBeside;
    p.bparts = (int32_t)(p.beside ? std::max<int64_t>(32, (tokens + 2047) / 2048 * 8) : std::max<int64_t>(1, std::min<int64_t>(256, tokens / 32)));
    p.bsum_bytes = (size_t)out * (p.bparts + 1) * 4;
    return p;
}

hipError_t launch_wgrad(int dtype, int grad_dtype, const Wgrad& a, hipStream_t st) {
    if (dtype == AL_DTYPE_BF16) return grad_dtype == AL_DTYPE_BF16 ? run<bf16, bf16>(a, st) : run<bf16, float>(a, st);
    return grad_dtype == AL_DTYPE_BF16 ? run<float, bf16>(a, st) : run<float, float>(a, st);
}

}  // namespace al
