// Token embeddings: the lookup with its scale, and the table's gradient summed in the order of the tokens sorted by id.
//
// Both are bound by memory: the lookup of 8192 x 2048 bf16 takes 10.3 us (67 MB), the gradient of 8192 tokens in 32000 x 4096 fp32 135 us (591 MB, the rows' kernel 107 at
// 5.5 TB/s). Small calls are bound by their launches: one token 6.2 us, 300 tokens in 5003 x 1001 21 us, three launches.
#include <algorithm>

#include "act_device.hpp"
#include "vocab_internal.hpp"

namespace al {

namespace {

__device__ __forceinline__ int64_t id_at(const Ids& ids, int64_t t) {
    return ids.wide ? static_cast<const int64_t*>(ids.p)[t] : (int64_t) static_cast<const int32_t*>(ids.p)[t];
}

// out[t] = scale table[id[t]], zeros for an id outside the table. A wavefront takes 512 columns of a token.
template <typename T, typename O>
__global__ __launch_bounds__(256) void lookup_kernel(Mat table, Ids ids, int64_t tokens, int64_t vocab, int32_t cols, int32_t parts, float scale, Mat out) {
    const int lane = threadIdx.x & 63;
    const int64_t total = tokens * parts, step = (int64_t)gridDim.x * 4;
    for (int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < total; i += step) {
        const int64_t t = i / parts;
        const int c = (int)(i - t * parts) * 512 + lane * 8;
        if (c >= cols) continue;
        const int64_t id = id_at(ids, t);
        float v[8] = {};
        if (id >= 0 && id < vocab) {
            Chunk<T> k;
            load_chunk(k, static_cast<const T*>(table.p) + id * table.ld, c, cols);
            k.get(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= scale;
        }
        store_chunk(static_cast<O*>(out.p) + t * out.ld, c, cols, v);
    }
}

constexpr uint64_t kNoToken = ~uint64_t(0);

// Runs of kSortRun keys (id, token) in order, each key put where as many of its run are less as it is from the run's begin. Ids outside the table come last. A workgroup
// places 64 keys of a run, a quarter of the run's keys compared by each wavefront: 1024^2 comparisons a run, but all of them at once (300 tokens 3.8 us, a bitonic
// network in registers 6.7; 8192 tokens 6.9 and 13.8). Up to 2^22 - 1 ids a key is 32 bits (the id, the place in the run).
template <typename K>
__global__ __launch_bounds__(256) void sort_kernel(Ids ids, int64_t tokens, int64_t vocab, uint64_t* keys) {
    constexpr bool kNarrow = sizeof(K) == 4;
    typedef K k16 __attribute__((ext_vector_type(16 / sizeof(K))));
    __shared__ __attribute__((aligned(16))) K s[kSortRun];
    __shared__ uint32_t below[4][64];
    const int64_t first = (int64_t)(blockIdx.x / (kSortRun / 64)) * kSortRun;
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, mine = (int)(blockIdx.x % (kSortRun / 64)) * 64 + lane;
    const int n = (int)std::min<int64_t>(kSortRun, tokens - first), quarter = (n + 31) / 32 * 8;
#pragma unroll
    for (int j = 0; j < kSortRun / 256; ++j) {
        const int p = j * 256 + threadIdx.x;
        const int64_t t = first + p, id = t < tokens ? id_at(ids, t) : -1;
        const uint64_t at = (uint64_t)(id >= 0 && id < vocab ? id : vocab);  // (keys stay different without a token)
        s[p] = t < tokens ? (K)(kNarrow ? at * kSortRun + (uint64_t)p : at << 32 | (uint64_t)t) : ~K(0);
    }
    __syncthreads();
    const K k = s[mine];
    uint32_t count = 0;
    for (int i = w * quarter; i < (w + 1) * quarter; i += 8) {
        k16 x[sizeof(K) / 2];
#pragma unroll
        for (int j = 0; j < (int)sizeof(K) / 2; ++j) x[j] = reinterpret_cast<const k16*>(s + i)[j];
#pragma unroll
        for (int j = 0; j < 8; ++j) count += x[j * (int)sizeof(K) / 16][j % (16 / (int)sizeof(K))] < k ? 1u : 0u;
    }
    below[w][lane] = count;
    __syncthreads();
    if (w || mine >= n) return;
    const uint64_t id = kNarrow ? (uint64_t)k / kSortRun : (uint64_t)k >> 32;
    keys[first + below[0][lane] + below[1][lane] + below[2][lane] + below[3][lane]] = id < (uint64_t)vocab ? id << 32 | (uint64_t)(first + mine) : kNoToken;
}

// Up to kMergeRuns sorted runs of `run` keys into one: a key's place is its own plus the numbers of the other runs' keys before it (keys without a
// token may be equal: those of an earlier run go first). The searches of 8 runs go on together, each halving its run.
constexpr int kMergeRuns = 64;
__global__ __launch_bounds__(256) void merge_kernel(const uint64_t* from, uint64_t* to, uint32_t tokens, uint32_t run, int steps) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= tokens) return;
    const uint32_t mine = i / run, group = mine / kMergeRuns * kMergeRuns;
    const uint64_t k = from[i];
    uint64_t place = (uint64_t)group * run + (i - mine * run);
    for (uint32_t o = group; o < group + kMergeRuns; o += 8) {
        if ((uint64_t)o * run >= tokens) break;
        uint32_t lo[8], n[8];  // n keys from lo on are still in question
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t at = (uint64_t)(o + j) * run;
            n[j] = at < tokens && o + j != mine ? std::min(run, (uint32_t)(tokens - at)) : 0u;
            lo[j] = at < tokens ? (uint32_t)at : 0u;
            place -= lo[j];
        }
        for (int s = 0; s < steps; ++s) {
            uint64_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = from[std::min(lo[j] + n[j] / 2, tokens - 1)];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool below = n[j] > 0 && (x[j] < k || (x[j] == k && o + j < mine));
                const uint32_t half = n[j] / 2;
                lo[j] += below ? half + 1 : 0u;
                n[j] = below ? n[j] - half - 1 : half;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) place += lo[j];
    }
    to[place] = k;
}

// A lane holds 4 columns in the sums, so that a wavefront's fp32 accesses are whole lines (8 would be two accesses of every other 16 bytes:
// 8192 tokens, 32000 x 4096 in fp32 251 us).
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
constexpr int kSlab = 1024;  // columns of a workgroup

// the 4 columns from c on of a row of `cols`, those past it 0
template <typename T>
struct Quad;
template <>
struct Quad<float> {
    f32x4 q;
    __device__ __forceinline__ void load(const float* row, int c, int cols) {
        if (c + 4 <= cols) {
            q = *reinterpret_cast<const f32x4_a4*>(row + c);
        } else {
            q = 0.0f;
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (c + j < cols) q[j] = row[c + j];
        }
    }
    __device__ __forceinline__ f32x4 get() const { return q; }
};
template <>
struct Quad<bf16> {
    u32x2 q;
    __device__ __forceinline__ void load(const bf16* row, int c, int cols) {
        if (c + 4 <= cols) {
            q = *reinterpret_cast<const u32x2_a2*>(row + c);
        } else {
            uint32_t h[3];
#pragma unroll
            for (int j = 0; j < 3; ++j) h[j] = c + j < cols ? row[c + j].b : 0u;
            q = u32x2{h[0] | h[1] << 16, h[2]};
        }
    }
    __device__ __forceinline__ f32x4 get() const {
        return f32x4{bits_f(q[0] << 16), bits_f(q[0] & 0xffff0000u), bits_f(q[1] << 16), bits_f(q[1] & 0xffff0000u)};
    }
};
// NT: past the caches (the rows' kernel, 8192 tokens, 32000 x 4096: 135 us, past the caches 109).
template <bool NT = false>
__device__ __forceinline__ void store4(float* row, int c, int cols, f32x4 v) {
    if (c + 4 <= cols) {
        if (NT)
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4_a4*>(row + c));
        else
            *reinterpret_cast<f32x4_a4*>(row + c) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (c + j < cols) row[c + j] = v[j];
}
template <bool NT = false>
__device__ __forceinline__ void store4(bf16* row, int c, int cols, f32x4 v) {
    if (c + 4 <= cols) {
        const u32x2 q = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (NT)
            __builtin_nontemporal_store(q, reinterpret_cast<u32x2_a2*>(row + c));
        else
            *reinterpret_cast<u32x2_a2*>(row + c) = q;
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (c + j < cols) put(row + c + j, v[j]);
}

// 4 columns of the sum over sorted tokens i0 .. i1, in order, the loads of 8 in flight.
template <typename T>
__device__ __forceinline__ void add_tokens(const EmbedBackward& a, int64_t i0, int64_t i1, int c, f32x4& s) {
    for (int64_t i = i0; i < i1; i += 8) {
        Quad<T> k[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < i1) k[j].load(static_cast<const T*>(a.dy.p) + (int64_t)(uint32_t)a.key0[i + j] * a.dy.ld, c, a.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < i1) s += k[j].get();
    }
}

// Two things that the sorted tokens give, side by side: sums over pieces of kPiece tokens of one id, so that of a frequent id's tokens one workgroup (for each kSlab columns of its row) is left
// with a sum for each kPiece, and
// for each row of the table where its tokens begin (a search by every lane; in the rows' own kernel it would hold up their stores: 8192 tokens, 32000 x 4096 in fp32 225 us).
template <typename T>
__global__ __launch_bounds__(256) void piece_kernel(EmbedBackward a, uint32_t pieces, uint32_t slabs) {
    if (blockIdx.x >= pieces * slabs) {
        const int64_t v = (int64_t)(blockIdx.x - pieces * slabs) * 256 + threadIdx.x;
        if (v > a.vocab) return;
        uint32_t lo = 0, n = (uint32_t)a.tokens;
        while (n > 0) {
            const uint32_t half = n / 2;
            if ((int64_t)(a.key0[lo + half] >> 32) < v)
                lo += half + 1, n -= half + 1;
            else
                n = half;
        }
        a.begin[v] = lo;
        return;
    }
    const uint32_t piece = blockIdx.x / slabs;
    const int64_t i0 = (int64_t)piece * kPiece;
    const uint32_t id = (uint32_t)(a.key0[i0] >> 32);
    if ((uint32_t)(a.key0[i0 + kPiece - 1] >> 32) != id || id >= (uint64_t)a.vocab) return;
    const int c = (int)(blockIdx.x % slabs) * kSlab + threadIdx.x * 4;
    if (c >= a.cols) return;
    f32x4 s = {};
    add_tokens<T>(a, i0, i0 + kPiece, c, s);
    store4(a.part + (int64_t)piece * a.cols, c, a.cols, s);
}

// kRows rows of the table's gradient, kSlab columns: sums of their tokens, scaled, added to the base and rounded once. 8 rows one after the other share the loads of
// where their tokens begin; 2 where there are too few rows for that to fill the device (300 tokens in 5003 x 1001: 10.9 and 8.8 us).
template <typename T, typename O, int kRows>
__global__ __launch_bounds__(256) void rows_kernel(EmbedBackward a) {
    const int64_t v0 = (int64_t)blockIdx.x * kRows;
    const int c = (int)blockIdx.y * kSlab + threadIdx.x * 4;
    if (c >= a.cols) return;
    const int rows = (int)std::min<int64_t>(kRows, a.vocab - v0);
    uint32_t begin[kRows + 1];
#pragma unroll
    for (int r = 0; r <= kRows; ++r) begin[r] = a.tokens > 0 ? a.begin[v0 + std::min(r, rows)] : 0u;
    for (int r = 0; r < rows; ++r) {
        const int64_t v = v0 + r;
        uint32_t i0 = begin[0], i1 = begin[1];
#pragma unroll
        for (int j = 0; j < kRows; ++j) begin[j] = begin[j + 1];
        if (i0 == i1 && a.base == a.dw) continue;
        f32x4 s = {};
        if (i0 < i1) {
            const int64_t p0 = ((int64_t)i0 + kPiece - 1) / kPiece, p1 = i1 / kPiece;
            const bool split = p0 < p1;
            add_tokens<T>(a, i0, split ? p0 * kPiece : i1, c, s);
            for (int64_t p = p0; p < p1; p += 8) {
                Quad<float> k[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (p + j < p1) k[j].load(a.part + (p + j) * a.cols, c, a.cols);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (p + j < p1) s += k[j].get();
            }
            if (split) add_tokens<T>(a, p1 * kPiece, i1, c, s);
            s *= a.scale;
        }
        if (a.base) {
            Quad<O> k;
            k.load(static_cast<const O*>(a.base) + v * a.cols, c, a.cols);
            s += k.get();
        }
        store4<true>(static_cast<O*>(a.dw) + v * a.cols, c, a.cols, s);
    }
}

template <typename T, typename O>
hipError_t run_lookup(Mat table, Ids ids, int64_t tokens, int64_t vocab, int32_t cols, float scale, Mat out, hipStream_t st) {
    const int32_t parts = (cols + 511) / 512;
    const int64_t blocks = std::min<int64_t>((tokens * parts + 3) / 4, 1 << 20);
    lookup_kernel<T, O><<<(uint32_t)blocks, 256, 0, st>>>(table, ids, tokens, vocab, cols, parts, scale, out);
    return hipGetLastError();
}

template <typename T, typename O>
hipError_t run_backward(EmbedBackward a, hipStream_t st) {
    const uint32_t slabs = (uint32_t)((a.cols + kSlab - 1) / kSlab);
    if (a.tokens > 0) {
        const uint32_t groups = (uint32_t)((a.tokens + 63) / 64);
        if (a.vocab < (1 << 22))
            sort_kernel<uint32_t><<<groups, 256, 0, st>>>(a.ids, a.tokens, a.vocab, a.key0);
        else
            sort_kernel<uint64_t><<<groups, 256, 0, st>>>(a.ids, a.tokens, a.vocab, a.key0);
        for (int64_t run = kSortRun; run < a.tokens; run *= kMergeRuns) {
            int steps = 1;  // a search among n keys takes floor(log2 n) + 1 steps
            while ((run >> steps) > 0) ++steps;
            merge_kernel<<<(uint32_t)((a.tokens + 255) / 256), 256, 0, st>>>(a.key0, a.key1, (uint32_t)a.tokens, (uint32_t)run, steps);
            std::swap(a.key0, a.key1);
        }
        const uint32_t pieces = (uint32_t)(a.tokens / kPiece);
        piece_kernel<T><<<pieces * slabs + (uint32_t)(a.vocab / 256 + 1), 256, 0, st>>>(a, pieces, slabs);
    }
    if (a.vocab * slabs >= 8 * 2048)
        rows_kernel<T, O, 8><<<dim3((uint32_t)((a.vocab + 7) / 8), slabs), 256, 0, st>>>(a);
    else
        rows_kernel<T, O, 2><<<dim3((uint32_t)((a.vocab + 1) / 2), slabs), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed_forward(int table_dtype, int out_dtype, Mat table, Ids ids, int64_t tokens, int64_t vocab, int32_t cols, float scale, Mat out,
                                hipStream_t st) {
    if (table_dtype == AL_DTYPE_BF16)
        return out_dtype == AL_DTYPE_BF16 ? run_lookup<bf16, bf16>(table, ids, tokens, vocab, cols, scale, out, st)
                                          : run_lookup<bf16, float>(table, ids, tokens, vocab, cols, scale, out, st);
    return out_dtype == AL_DTYPE_BF16 ? run_lookup<float, bf16>(table, ids, tokens, vocab, cols, scale, out, st)
                                      : run_lookup<float, float>(table, ids, tokens, vocab, cols, scale, out, st);
}

EmbedPlan embed_plan(int64_t tokens, int64_t vocab, int64_t cols) {
    const auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
    EmbedPlan p = {};
    p.key1_off = up((size_t)tokens * 8);
    p.begin_off = p.key1_off + (tokens > kSortRun ? up((size_t)tokens * 8) : 0);
    p.part_off = p.begin_off + (tokens > 0 ? up((size_t)(vocab + 1) * 4) : 0);
    p.bytes = p.part_off + up((size_t)(tokens / kPiece) * cols * 4);
    return p;
}

hipError_t launch_embed_backward(int dtype, int grad_dtype, const EmbedBackward& a, hipStream_t st) {
    if (dtype == AL_DTYPE_BF16) return grad_dtype == AL_DTYPE_BF16 ? run_backward<bf16, bf16>(a, st) : run_backward<bf16, float>(a, st);
    return grad_dtype == AL_DTYPE_BF16 ? run_backward<float, bf16>(a, st) : run_backward<float, float>(a, st);
}

}  // namespace al
