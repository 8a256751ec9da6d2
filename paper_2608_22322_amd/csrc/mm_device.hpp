// Products of 16-bit matrices on the matrix cores with a fused end: the core that the orthogonalised update and the
// linear head share.
//
//   out[m][n] = sum over k of A(m, k) B(n, k)
//
// Either operand lies in memory with k along its rows (a row for each m or n) or with k down its rows (a row for each
// k), and is one matrix of 16-bit numbers or the sum of a high and a low part (products of two low parts are dropped). Sums
// are fp32. k is taken in turns of 64, and where B ends inside a turn A holds zeros.
#pragma once

#include <type_traits>

#include "act_device.hpp"

namespace al {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 MmAcc;

constexpr int kMmTurn = 64;

// An operand of 16-bit values. k along the rows: `rows` rows of `cols` values each; k down the rows: `rows` values of k, each a row
// of `cols`. What a tile reaches past either is read from the last row or the last 8 columns instead (cols is a multiple of
// 8, ld too, and p is 16-byte aligned), for outputs that are not written or, by MmEnds, against zeros of the other operand.
struct MmOperand {
    const uint16_t* p;
    int64_t lo;  // elements from the high part to the low
    int32_t ld, rows, cols;
};

// Where B's k may end inside a turn: nowhere; what is past the end is the last there is, finite, against A's zeros; or (k along the rows, B of any values: an infinity against a zero would be a
// NaN) it is A's last 8 columns of its first row, which are zeros then.
enum MmEnds : int { kMmWhole, kMmLast, kMmZeros };

struct Mm {
    MmOperand a, b;
    int32_t m, n, turns;
    // Operands in parts are taken together by 64-wide tiles (PA, PB: their parts; what is loaded serves two or three products). Larger tiles, whose turns of one part already are 32 and 64 KB (two
    // parts of both operands would leave one 128-wide workgroup to a compute unit, and a 256-wide one no second turn), take
    // `segs` segments of `turns` turns each instead, segment i with the low part of A (B) where bit i of amask (bmask) is set.
    int32_t segs;
    uint32_t amask, bmask;
    int32_t splits;  // over the turns of all segments
    int32_t sym;     // A A^T: the tiles on and below the diagonal alone
    float* part;     // splits > 1: partial sums, [split][tile][lanes' order]
};

// A workgroup's tile of B x B outputs. PA, PB: parts of the operands.
template <int B>
struct MmTile {
    static constexpr int kThreads = B == 256 ? 512 : 256, kWaves = kThreads / 64, WM = B / 2, WN = B == 64 ? 32 : 64, FM = WM / 16, FN = WN / 16;
    static constexpr int kChunks = B * kMmTurn / 8 / kThreads;  // 16-byte pieces of a part that a thread stages in a turn
    static __device__ __forceinline__ int wave_m(int w) { return w / (B / WN) * WM; }
    static __device__ __forceinline__ int wave_n(int w) { return w % (B / WN) * WN; }
    static uint32_t side(int n) { return (uint32_t)((n + B - 1) / B); }
    static uint32_t tiles(const Mm& p) { return side(p.m) * side(p.n); }
};
// Turns that LDS holds: 64 KB of them, two workgroups a compute unit, or two turns of 256-wide tiles (128 KB).
template <int B, int PA, int PB>
constexpr int mm_stages() { return B == 64 && PA + PB == 2 ? 4 : 2; }

// The places of a tile's turns: arrays of their own, so that the compiler knows that a read of one does not wait for the loads into the others.
template <int PA, int PB, int S>
struct MmPlaces {
    uint16_t *a[S][PA], *b[S][PB];
};
#define MM_ARRAY(name, used) __shared__ __attribute__((aligned(16))) uint16_t name[(used) ? kMmArray : 8]
#define MM_PLACES(B, PA, PB, places)                                                                                               \
    constexpr int kMmArray = (B) * kMmTurn, kMmStages = mm_stages<B, PA, PB>();                                                    \
    MM_ARRAY(mm_a00, true); MM_ARRAY(mm_a10, true); MM_ARRAY(mm_b00, true); MM_ARRAY(mm_b10, true);                                \
    MM_ARRAY(mm_a01, PA > 1); MM_ARRAY(mm_a11, PA > 1); MM_ARRAY(mm_b01, PB > 1); MM_ARRAY(mm_b11, PB > 1);                        \
    MM_ARRAY(mm_a20, kMmStages > 2); MM_ARRAY(mm_a30, kMmStages > 2); MM_ARRAY(mm_b20, kMmStages > 2); MM_ARRAY(mm_b30, kMmStages > 2); \
    MmPlaces<PA, PB, kMmStages> places;                                                                                            \
    places.a[0][0] = mm_a00, places.a[1][0] = mm_a10, places.b[0][0] = mm_b00, places.b[1][0] = mm_b10;                            \
    if constexpr (PA > 1) places.a[0][PA - 1] = mm_a01, places.a[1][PA - 1] = mm_a11;                                              \
    if constexpr (PB > 1) places.b[0][PB - 1] = mm_b01, places.b[1][PB - 1] = mm_b11;                                              \
    if constexpr (kMmStages > 2)                                                                                                   \
        places.a[kMmStages - 2][0] = mm_a20, places.a[kMmStages - 1][0] = mm_a30, places.b[kMmStages - 2][0] = mm_b20, places.b[kMmStages - 1][0] = mm_b30

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

// Sums of 16 x 16 blocks: a lane holds row 16 i + l % 16 and columns 16 j + 4 (l / 16) + 0..3 of its wavefront's part. AK, BK: k along the rows of the operand.
template <class T, int B, bool AK, bool BK, int ENDS, int PA, int PB>
struct MmCore {
    typedef MmTile<B> G;
    typedef __attribute__((address_space(3))) uint16_t* lds_t;
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    static constexpr int S = mm_stages<B, PA, PB>();
    typedef MmPlaces<PA, PB, S> Places;

    // k of a piece within its turn, k along the rows
    static __device__ __forceinline__ int column(int q) { return ((q & 7) ^ ((q >> 3) & 7)) * 8; }
    // byte offset of this thread's piece i of the turn at k0 from the turn's first element. SHORT: the operand may end inside the turn.
    template <bool K, bool SHORT>
    static __device__ __forceinline__ uint32_t offset(const MmOperand& o, int first, int i, int tid, int k0) {
        const int q = i * G::kThreads + tid;
        if (K) {
            const int r = q >> 3, c = column(q);
            return (uint32_t)(min(first + r, o.rows - 1) - first) * (uint32_t)o.ld * 2u + (uint32_t)(SHORT ? min(k0 + c, o.cols - 8) - k0 : c) * 2u;
        }
        const int k = q / (B / 8), s = q % (B / 8), c = (((s >> 1) ^ mm_swizzle<B>(k)) << 4) | ((s & 1) << 3);
        return (uint32_t)(SHORT ? min(k0 + k, o.rows - 1) - k0 : k) * (uint32_t)o.ld * 2u + (uint32_t)(min(first + c, o.cols - 8) - first) * 2u;
    }

    template <bool K, int SHORT>
    static __device__ __forceinline__ void issue(const MmOperand& o, const uint16_t* p, int first, int k0, const uint32_t (&off)[G::kChunks], uint16_t* lds,
                                                 int tid, const uint16_t* zeros = nullptr) {
        const char* const at = reinterpret_cast<const char*>(K ? p + (int64_t)first * o.ld + k0 : p + (int64_t)k0 * o.ld + first);
        uint16_t* const to = lds + (tid & ~63) * 8;
#pragma unroll
        for (int i = 0; i < G::kChunks; ++i) {
            static_assert(K || SHORT != kMmZeros, "");
            const uint32_t f = SHORT == kMmLast ? offset<K, true>(o, first, i, tid, k0) : off[i];
            const char* const from = SHORT == kMmZeros && k0 + column(i * G::kThreads + tid) >= o.cols ? reinterpret_cast<const char*>(zeros) : at + f;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                             (__attribute__((address_space(3))) void*)(to + i * G::kThreads * 8), 16, 0, 0);
        }
    }

    // A lane's places of block 0, in bytes: of either half (k along the rows), or of the two reads of a fragment (k down the rows, where
    // block i's unit differs from block 0's by an exclusive or).
    template <bool K>
    struct Reader {
        uint32_t at[2];
        __device__ __forceinline__ Reader(int first, int lane) {
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

    // Turns t0 .. t1 of the tile whose first output is m0, n0.
    static __device__ __forceinline__ void run(const Mm& p, int m0, int n0, int t0, int t1, const Places& at, MmAcc (&acc)[G::FM][G::FN]) {
        const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
        uint32_t oa[G::kChunks], ob[G::kChunks];
#pragma unroll
        for (int i = 0; i < G::kChunks; ++i) {
            oa[i] = offset<AK, false>(p.a, m0, i, tid, 0);
            ob[i] = offset<BK, false>(p.b, n0, i, tid, 0);
        }
        int seg = t0 / p.turns, k0 = (t0 - seg * p.turns) * kMmTurn;  // of the next turn to load
        const auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < PA; ++q) issue<AK, kMmWhole>(p.a, q || (p.amask >> seg) & 1 ? p.a.p + p.a.lo : p.a.p, m0, k0, oa, at.a[s][q], (w << 6) | lane);
#pragma unroll
            for (int q = 0; q < PB; ++q) issue<BK, ENDS>(p.b, q || (p.bmask >> seg) & 1 ? p.b.p + p.b.lo : p.b.p, n0, k0, ob, at.b[s][q], (w << 6) | lane, p.a.p + (p.a.cols - 8));
            k0 += kMmTurn;
            if (k0 == p.turns * kMmTurn) k0 = 0, ++seg;
        };
        Reader<AK> am(G::wave_m(w), lane);
        Reader<BK> bn(G::wave_n(w), lane);
        struct Half {
            MmFragment a[PA][G::FM], b[PB][G::FN];
        };
        const auto read_a = [&](Half& f, int s, int i, int h) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < PA; ++q) f.a[q][i] = am.read(at.a[s][q], i, h);
        };
        const auto read_b = [&](Half& f, int s, int h) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < PB; ++q)
#pragma unroll
                for (int j = 0; j < G::FN; ++j) f.b[q][j] = bn.read(at.b[s][q], j, h);
        };
        const auto multiply = [&](const Half& f, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < G::FN; ++j) acc[i][j] = mm_mul<T>(f.b[0][j], f.a[0][i], acc[i][j]);
            if (PB > 1)
#pragma unroll
                for (int j = 0; j < G::FN; ++j) acc[i][j] = mm_mul<T>(f.b[PB - 1][j], f.a[0][i], acc[i][j]);
            if (PA > 1)
#pragma unroll
                for (int j = 0; j < G::FN; ++j) acc[i][j] = mm_mul<T>(f.b[0][j], f.a[PA - 1][i], acc[i][j]);
        };
        // This wavefront's pieces of a turn have arrived (`behind`: those of the S - 2 turns after it may be in flight: vmcnt), and what it read of an earlier one is
        // in its registers (lgkmcnt); behind the barrier that holds for all, and the loads into the earlier turn's place may begin. (__syncthreads would wait for every load.)
        const auto meet = [&](bool behind) __attribute__((always_inline)) {
            if (S > 2 && behind)
                __builtin_amdgcn_s_waitcnt(0x0070 | (S - 2) * (PA + PB) * G::kChunks);
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
            // cover them with, and take longer so).
            Half f0, f1;
            const auto read = [&](Half& f, int s, int h) __attribute__((always_inline)) {
                am.renew();
                bn.renew();
                read_b(f, s, h);
#pragma unroll
                for (int i = 0; i < G::FM; ++i) read_a(f, s, i, h);
            };
            const auto multiply_all = [&](const Half& f) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < G::FM; ++i) multiply(f, i);
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
                    multiply_all(f0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (t + s + 1 < t1) {
                        meet(t + s + S - 1 < t1);
                        read(f0, (s + 1) % S, 0);
                        if (t + s + S < t1) load(s);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    multiply_all(f1);
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
                        Half f;
                        read_b(f, s, h);
#pragma unroll
                        for (int i = 0; i < G::FM; ++i) {
                            read_a(f, s, i, h);
                            multiply(f, i);
                        }
                    }
                }
            }
        }
    }
};

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

// E: end(row, first column, 4 sums) takes 4 neighbouring outputs. One with E::kRows takes all of a lane's rows instead (every 16th from `row` on),
// end.rows<FM, FN>(row, first column of its part, lane, sums), and no splits.
template <class E, class = void>
struct MmRows : std::false_type {};
template <class E>
struct MmRows<E, std::enable_if_t<E::kRows>> : std::true_type {};

template <class T, int B, bool AK, bool BK, int ENDS, int PA, class E>
__global__ __launch_bounds__(MmTile<B>::kThreads, 2) void mm_kernel(Mm p, E end) {
    typedef MmTile<B> G;
    MM_PLACES(B, PA, 1, places);
    const MmId id = mm_id<B>(p);
    const int64_t turns = p.turns * p.segs;
    const int t0 = (int)(turns * id.split / p.splits), t1 = (int)(turns * (id.split + 1) / p.splits);
    MmAcc acc[G::FM][G::FN] = {};
    MmCore<T, B, AK, BK, ENDS, PA, 1>::run(p, id.m * B, id.n * B, t0, t1, places, acc);
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
    if constexpr (MmRows<E>::value) {
        end.template rows<G::FM, G::FN>(m, n, lane, acc);
    } else {
#pragma unroll
        for (int i = 0; i < G::FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < G::FN; ++j) end(m + 16 * i, n + 16 * j, acc[i][j]);
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

// B in one part.
template <class T, int B, bool AK, bool BK, int ENDS, int PA, class E>
hipError_t mm_launch(const Mm& p, const E& end, hipStream_t st) {
    const uint32_t tiles = MmTile<B>::tiles(p);
    if (tiles == 0) return hipSuccess;
    mm_kernel<T, B, AK, BK, ENDS, PA, E><<<tiles * (uint32_t)p.splits, MmTile<B>::kThreads, 0, st>>>(p, end);
    if constexpr (!MmRows<E>::value)
        if (p.splits > 1) mm_join_kernel<B, E><<<tiles * (B * B / 1024), 256, 0, st>>>(p, end, tiles);
    return hipGetLastError();
}

}  // namespace al
