// Products of 16-bit matrices on the matrix cores with a fused end: the core that the orthogonalised update and the
// linear head share.
//
//   out[m][n] = sum over k of A(m, k) B(n, k)
//
// Either operand lies in memory with k along its rows (a row for each m or n) or with k down its rows (a row for each
// k). Sums are fp32. k is taken in turns of 64, and where an operand ends inside a turn the other one holds zeros.
#pragma once

#include <type_traits>

#include "act_device.hpp"

namespace al {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMmTurn = 64;

// An operand of 16-bit values. k along the rows: `rows` rows of `cols` values each; k down the rows: `rows` values of k, each a row
// of `cols`. What a tile reaches past either is read from the last row or the last 8 columns instead (cols is a multiple of
// 8, ld too, and p is 16-byte aligned), for outputs that are not written or against zeros of the other operand.
struct MmOperand {
    const uint16_t* p;
    int64_t lo;  // elements from a matrix to its low part
    int32_t ld, rows, cols;
};

// A product. An operand may be the sum of a high and a low part: `segs` segments of `turns` turns each, segment
// i with the low part of A (B) where bit i of amask (bmask) is set.
struct Mm {
    MmOperand a, b;
    int32_t m, n, turns, segs;
    uint32_t amask, bmask;
    int32_t splits;  // over the turns
    int32_t sym;     // A A^T: the tiles on and below the diagonal alone
    float* part;     // splits > 1: partial sums, [split][tile][lanes' order]
};

template <int B>
struct MmTile {
    static constexpr int kThreads = B == 256 ? 512 : 256, kWaves = kThreads / 64, WM = B / 2, WN = B == 64 ? 32 : 64, FM = WM / 16, FN = WN / 16;
    static constexpr int kStages = B == 64 ? 4 : 2;  // turns in LDS: 64 (64-wide tiles), 64 and 128 KB
    static constexpr int kChunks = B * kMmTurn / 8 / kThreads;  // 16-byte pieces of an operand that a thread stages in a turn
    static __device__ __forceinline__ int wave_m(int w) { return w / (B / WN) * WM; }
    static __device__ __forceinline__ int wave_n(int w) { return w % (B / WN) * WN; }
    static uint32_t side(int n) { return (uint32_t)((n + B - 1) / B); }
    static uint32_t tiles(const Mm& p) { return side(p.m) * side(p.n); }
};

typedef f32x4 MmAcc;

union MmFragment {
    s16x4 h[2];
    u32x4 q;
    bf16x8 b;
    f16x8 f;
};
template <class T>
__device__ __forceinline__ MmAcc mm_mul(const MmFragment& x, const MmFragment& y, MmAcc c) {
    if constexpr (std::is_same<T, bf16>::value)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.b, y.b, c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(x.f, y.f, c, 0, 0, 0);
}

// An operand's turn in LDS, in 16-byte pieces that the loads put there in the threads' order.
// k along the rows: 8 pieces a row, piece c of row r at c ^ r % 8: eight lanes that read one piece of 8 rows meet all banks.
// k down the rows: B / 8 pieces a row; 32-byte units are exchanged by the row so that the 8 rows that half a wavefront reads
// at once (k = 8 g + 0..3, two g) lie in different banks.
template <int B>
__device__ __forceinline__ int mm_swizzle(int k) {
    if (B == 64) return ((k >> 1) & 1) | ((k >> 2) & 2);
    return ((k & 3) | ((k >> 1) & 4) | ((k << 1) & 8)) & (B / 16 - 1);
}

// Sums of 16 x 16 blocks: a lane holds row 16 i + l % 16 and columns 16 j + 4 (l / 16) + 0..3 of its wavefront's part.
template <class T, int B, bool AK, bool BK, bool ENDS>
struct MmCore {
    typedef MmTile<B> G;
    typedef __attribute__((address_space(3))) uint16_t* lds_t;
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

    // byte offset of this thread's piece i of the turn at k0 from the turn's first element. SHORT: the operand may end inside the turn.
    template <bool K, bool SHORT>
    static __device__ __forceinline__ uint32_t offset(const MmOperand& o, int first, int i, int tid, int k0) {
        const int q = i * G::kThreads + tid;
        if (K) {
            const int r = q >> 3, c = ((q & 7) ^ (r & 7)) * 8;
            return (uint32_t)(min(first + r, o.rows - 1) - first) * (uint32_t)o.ld * 2u + (uint32_t)(SHORT ? min(k0 + c, o.cols - 8) - k0 : c) * 2u;
        }
        const int k = q / (B / 8), s = q % (B / 8), c = (((s >> 1) ^ mm_swizzle<B>(k)) << 4) | ((s & 1) << 3);
        return (uint32_t)(SHORT ? min(k0 + k, o.rows - 1) - k0 : k) * (uint32_t)o.ld * 2u + (uint32_t)(min(first + c, o.cols - 8) - first) * 2u;
    }

    template <bool K, bool SHORT>
    static __device__ __forceinline__ void issue(const MmOperand& o, const uint16_t* p, int first, int k0, const uint32_t (&off)[G::kChunks], uint16_t* lds,
                                                 int tid) {
        const char* const at = reinterpret_cast<const char*>(K ? p + (int64_t)first * o.ld + k0 : p + (int64_t)k0 * o.ld + first);
        uint16_t* const to = lds + (tid & ~63) * 8;
#pragma unroll
        for (int i = 0; i < G::kChunks; ++i) {
            const uint32_t f = SHORT ? offset<K, SHORT>(o, first, i, tid, k0) : off[i];
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(at + f),
                                             (__attribute__((address_space(3))) void*)(to + i * G::kThreads * 8), 16, 0, 0);
        }
    }

    // A lane's places of block 0, in bytes: of either half (k along the rows), or of the two reads of a fragment (k down the rows, where
    // block i's unit differs from block 0's by an exclusive or).
    template <bool K>
    struct Places {
        uint32_t at[2];
        __device__ __forceinline__ Places(int first, int lane) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (K) {
                    at[s] = (uint32_t)((first + (lane & 15)) * kMmTurn + (((4 * s + (lane >> 4)) ^ (lane & 7)) << 3)) * 2u;
                } else {
                    const int k = 8 * (lane >> 4) + 4 * s + ((lane >> 2) & 3);
                    at[s] = (uint32_t)(k * B + (((first / 16) ^ mm_swizzle<B>(k)) << 4) + 4 * (lane & 3)) * 2u;
                }
            }
        }
        // (The blocks' places are formed anew in each turn: kept in registers they would push sums out of them.)
        __device__ __forceinline__ void renew() {
            if (!K) asm volatile("" : "+v"(at[0]), "+v"(at[1]));
        }
        __device__ __forceinline__ MmFragment read(const uint16_t* lds, int i, int h) const {
            const char* const base = reinterpret_cast<const char*>(lds);
            MmFragment f;
            if (K) {
                f.q = *reinterpret_cast<const u32x4*>(base + at[h] + i * 32 * kMmTurn);
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    f.h[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds_t)(uint16_t*)(base + (at[s] ^ (uint32_t)(i << 5)) + h * 64 * B));
            }
            return f;
        }
    };

    // Turns t0 .. t1 of a tile. as, bs: kStages places for a turn of either operand (arrays of their own, so that the compiler knows that a
    // read of one does not wait for the loads into the others).
    static __device__ __forceinline__ void run(const Mm& p, int m0, int n0, int t0, int t1, uint16_t* const (&as)[G::kStages],
                                               uint16_t* const (&bs)[G::kStages], MmAcc (&acc)[G::FM][G::FN]) {
        constexpr int S = G::kStages;
        const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
        uint32_t oa[G::kChunks], ob[G::kChunks];
#pragma unroll
        for (int i = 0; i < G::kChunks; ++i) {
            oa[i] = offset<AK, false>(p.a, m0, i, tid, 0);
            ob[i] = offset<BK, false>(p.b, n0, i, tid, 0);
        }
        const uint16_t *const pa = p.a.p, *const pb = p.b.p;
        int seg = t0 / p.turns, k0 = (t0 - seg * p.turns) * kMmTurn;  // of the next turn to load
        const auto load = [&](int s) __attribute__((always_inline)) {
            issue<AK, false>(p.a, (p.amask >> seg) & 1 ? pa + p.a.lo : pa, m0, k0, oa, as[s], (w << 6) | lane);
            issue<BK, ENDS>(p.b, (p.bmask >> seg) & 1 ? pb + p.b.lo : pb, n0, k0, ob, bs[s], (w << 6) | lane);
            k0 += kMmTurn;
            if (k0 == p.turns * kMmTurn) k0 = 0, ++seg;
        };
        Places<AK> am(G::wave_m(w), lane);
        Places<BK> bn(G::wave_n(w), lane);
        // This wavefront's pieces of a turn have arrived (`behind`: those of the S - 2 turns after it may be in flight: vmcnt), and what it read of an earlier one is
        // in its registers (lgkmcnt); behind the barrier that holds for all, and the loads into the earlier turn's place may begin. (__syncthreads would wait for every load.)
        const auto meet = [&](bool behind) __attribute__((always_inline)) {
            if (S > 2 && behind)
                __builtin_amdgcn_s_waitcnt(0x0070 | (S - 2) * 2 * G::kChunks);
            else
                __builtin_amdgcn_s_waitcnt(0x0070);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        if (t0 >= t1) return;
        if constexpr (B == 256) {
            // The barrier lies between the halves of a turn: the products of the second half, whose fragments are in registers, cover the next turn's first
            // reads and the issuing of loads (8 wavefronts, 2 a SIMD; 4096^3: 240 us with the barrier between the turns, 220 so. The smaller tiles have fewer products to
            // cover them with, and take longer so.)
            struct Half {
                MmFragment a[G::FM], b[G::FN];
            } f0, f1;
            const auto read = [&](Half& f, int s, int h) __attribute__((always_inline)) {
                am.renew();
                bn.renew();
#pragma unroll
                for (int j = 0; j < G::FN; ++j) f.b[j] = bn.read(bs[s], j, h);
#pragma unroll
                for (int i = 0; i < G::FM; ++i) f.a[i] = am.read(as[s], i, h);
            };
            const auto multiply = [&](const Half& f) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < G::FM; ++i)
#pragma unroll
                    for (int j = 0; j < G::FN; ++j) acc[i][j] = mm_mul<T>(f.b[j], f.a[i], acc[i][j]);
            };
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (t0 + s < t1) load(s);
            meet(false);
            read(f0, 0, 0);
            for (int t = t0; t < t1; t += S) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    if (t + s >= t1) break;
                    read(f1, s, 1);
                    __builtin_amdgcn_sched_barrier(0);
                    multiply(f0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (t + s + 1 < t1) {
                        meet(t + s + S - 1 < t1);
                        read(f0, (s + 1) % S, 0);
                        if (t + s + S < t1) load(s);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    multiply(f1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
#pragma unroll
            for (int s = 0; s < S - 1; ++s)
                if (t0 + s < t1) load(s);
            for (int t = t0; t < t1; t += S) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    if (t + s >= t1) break;
                    meet(t + s + S - 2 < t1);
                    if (t + s + S - 1 < t1) load((s + S - 1) % S);
                    am.renew();
                    bn.renew();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        MmFragment fb[G::FN];
#pragma unroll
                        for (int j = 0; j < G::FN; ++j) fb[j] = bn.read(bs[s], j, h);
#pragma unroll
                        for (int i = 0; i < G::FM; ++i) {
                            const MmFragment fa = am.read(as[s], i, h);
#pragma unroll
                            for (int j = 0; j < G::FN; ++j) acc[i][j] = mm_mul<T>(fb[j], fa, acc[i][j]);
                        }
                    }
                }
            }
        }
    }
};

// The places of a tile's turns in LDS: arrays of their own.
#define MM_PLACES(B, as, bs)                                                                                                                        \
    __shared__ __attribute__((aligned(16))) uint16_t as##0_[B * kMmTurn], as##1_[B * kMmTurn], bs##0_[B * kMmTurn], bs##1_[B * kMmTurn];            \
    __shared__ __attribute__((aligned(16))) uint16_t as##2_[MmTile<B>::kStages > 2 ? B * kMmTurn : 8], as##3_[MmTile<B>::kStages > 2 ? B * kMmTurn : 8], \
        bs##2_[MmTile<B>::kStages > 2 ? B * kMmTurn : 8], bs##3_[MmTile<B>::kStages > 2 ? B * kMmTurn : 8];                                         \
    uint16_t *as[MmTile<B>::kStages], *bs[MmTile<B>::kStages];                                                                                      \
    as[0] = as##0_, as[1] = as##1_, bs[0] = bs##0_, bs[1] = bs##1_;                                                                                 \
    if constexpr (MmTile<B>::kStages > 2) as[2] = as##2_, as[3] = as##3_, bs[2] = bs##2_, bs[3] = bs##3_

// Tile number (the same in all lanes) -> its rows and columns of tiles: the triangle on and below the diagonal row by row, others in bands of 8 along m.
struct MmAt {
    int m, n;
};
template <int B>
__device__ __forceinline__ MmAt mm_at(const Mm& p, uint32_t tile) {
    if (p.sym) {
        uint32_t i = (uint32_t)((sqrtf(8.0f * (float)tile + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > tile) --i;
        while ((i + 1) * (i + 2) / 2 <= tile) ++i;
        return {__builtin_amdgcn_readfirstlane((int)i), __builtin_amdgcn_readfirstlane((int)(tile - i * (i + 1) / 2))};
    }
    const uint32_t mt = (uint32_t)((p.m + B - 1) / B), nt = (uint32_t)((p.n + B - 1) / B);
    const uint32_t band = tile / (8 * nt), rows = min(8u, mt - band * 8), q = tile - band * 8 * nt, n = q / rows;
    return {__builtin_amdgcn_readfirstlane((int)(band * 8 + q - n * rows)), __builtin_amdgcn_readfirstlane((int)n)};
}

// Workgroup -> split and tile; an XCD takes a contiguous share.
struct MmId : MmAt {
    int split, tile;
};
template <int B>
__device__ __forceinline__ MmId mm_id(const Mm& p) {
    const uint32_t per = gridDim.x / (uint32_t)p.splits, id = xcd_block(blockIdx.x, gridDim.x), s = id / per;
    MmId t;
    t.split = (int)s;
    t.tile = (int)(id - s * per);
    static_cast<MmAt&>(t) = mm_at<B>(p, (uint32_t)t.tile);
    return t;
}

// E: end(row, first column, 4 sums) takes 4 neighbouring outputs. One with E::kRows takes a wavefront's
// row instead, end.row<FN>(row, first column of its part, lane, sums), and no splits.
template <class E, class = void>
struct MmRows : std::false_type {};
template <class E>
struct MmRows<E, std::enable_if_t<E::kRows>> : std::true_type {};
template <class T, int B, bool AK, bool BK, bool ENDS, class E>
__global__ __launch_bounds__(MmTile<B>::kThreads, 2) void mm_kernel(Mm p, E end) {
    typedef MmTile<B> G;
    MM_PLACES(B, as, bs);
    const MmId id = mm_id<B>(p);
    const int total = p.turns * p.segs, t0 = (int)((int64_t)total * id.split / p.splits), t1 = (int)((int64_t)total * (id.split + 1) / p.splits);
    MmAcc acc[G::FM][G::FN] = {};
    MmCore<T, B, AK, BK, ENDS>::run(p, id.m * B, id.n * B, t0, t1, as, bs, acc);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int m = id.m * B + G::wave_m(w) + (lane & 15), n = id.n * B + G::wave_n(w) + 4 * (lane >> 4);
    if (p.splits > 1) {
        f32x4* const part = reinterpret_cast<f32x4*>(p.part) + (((int64_t)id.split * (gridDim.x / (uint32_t)p.splits) + id.tile) * G::kWaves + w) * (G::FM * G::FN * 64) + lane;
#pragma unroll
        for (int i = 0; i < G::FM; ++i)
#pragma unroll
            for (int j = 0; j < G::FN; ++j) part[(i * G::FN + j) * 64] = acc[i][j];
        return;
    }
#pragma unroll
    for (int i = 0; i < G::FM; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MmRows<E>::value) {
            end.template row<G::FN>(m + 16 * i, n, lane, acc[i]);
            continue;
        }
#pragma unroll
        for (int j = 0; j < G::FN; ++j) {
            if constexpr (!MmRows<E>::value) end(m + 16 * i, n + 16 * j, acc[i][j]);
        }
    }
}

// The splits' partial sums, added in order.
template <int B, class E>
__global__ __launch_bounds__(256) void mm_join_kernel(Mm p, E end, uint32_t tiles) {
    typedef MmTile<B> G;
    constexpr uint32_t kBlocks = B * B / 1024;
    const uint32_t tile = blockIdx.x / kBlocks, at = blockIdx.x % kBlocks * 256 + threadIdx.x, lane = at & 63, slot = at >> 6;
    const int64_t size = (int64_t)tiles * (B * B / 4);
    const f32x4* q = reinterpret_cast<const f32x4*>(p.part) + (int64_t)tile * (B * B / 4) + at;
    f32x4 v = {};
    int s = 0;
    for (; s + 4 <= p.splits; s += 4, q += 4 * size) {
        f32x4 t[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) t[r] = q[r * size];
#pragma unroll
        for (int r = 0; r < 4; ++r) v += t[r];
    }
    for (; s < p.splits; ++s, q += size) v += *q;
    const uint32_t w = slot / (G::FM * G::FN), e = slot % (G::FM * G::FN);
    const MmAt id = mm_at<B>(p, tile);
    end(id.m * B + G::wave_m((int)w) + (int)(lane & 15) + 16 * (int)(e / G::FN), id.n * B + G::wave_n((int)w) + 4 * (int)(lane >> 4) + 16 * (int)(e % G::FN), v);
}

template <class T, int B, bool AK, bool BK, bool ENDS, class E>
hipError_t mm_launch(const Mm& p, const E& end, hipStream_t st) {
    const uint32_t tiles = MmTile<B>::tiles(p);
    if (tiles == 0) return hipSuccess;
    mm_kernel<T, B, AK, BK, ENDS, E><<<tiles * (uint32_t)p.splits, MmTile<B>::kThreads, 0, st>>>(p, end);
    if constexpr (!MmRows<E>::value)
        if (p.splits > 1) mm_join_kernel<B, E><<<tiles * (B * B / 1024), 256, 0, st>>>(p, end, tiles);
    return hipGetLastError();
}

}  // namespace al
