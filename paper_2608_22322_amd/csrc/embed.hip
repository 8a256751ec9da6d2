// Token embeddings: the lookup with its scale, and the table's gradient summed in the order of the tokens sorted by id.
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

// Runs of kSortRun keys (id, token), each sorted by a workgroup in LDS (a bitonic network; keys differ, so their order is one). Ids outside the table come last.
__global__ __launch_bounds__(1024) void sort_kernel(Ids ids, int64_t tokens, int64_t vocab, uint64_t* keys) {
    __shared__ uint64_t s[kSortRun];
    const int64_t first = (int64_t)blockIdx.x * kSortRun;
    for (int i = threadIdx.x; i < kSortRun; i += 1024) {
        const int64_t t = first + i;
        const int64_t id = t < tokens ? id_at(ids, t) : -1;
        s[i] = id >= 0 && id < vocab ? (uint64_t)id << 32 | (uint64_t)t : kNoToken - (uint64_t)(kSortRun - 1 - i);
    }
    __syncthreads();
    for (int size = 2; size <= kSortRun; size *= 2) {
        for (int gap = size / 2; gap > 0; gap /= 2) {
            for (int i = threadIdx.x; i < kSortRun / 2; i += 1024) {
                const int a = (i & ~(gap - 1)) * 2 + (i & (gap - 1)), b = a + gap;
                const uint64_t x = s[a], y = s[b];
                if ((x > y) == ((a & size) == 0)) s[a] = y, s[b] = x;
            }
            __syncthreads();
        }
    }
    for (int i = threadIdx.x; i < kSortRun; i += 1024)
        if (first + i < tokens) keys[first + i] = s[i];
}

// Pairs of sorted runs of `run` keys into one: a key's place is its own plus the number of the other run's keys before it.
__global__ __launch_bounds__(256) void merge_kernel(const uint64_t* from, uint64_t* to, int64_t tokens, int64_t run) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= tokens) return;
    const int64_t mine = i / run, pair = mine & ~int64_t(1), other = mine ^ 1, o0 = std::min(other * run, tokens), o1 = std::min(o0 + run, tokens);
    const uint64_t k = from[i];
    // (keys without a token may be equal: those of the first run go first)
    int64_t lo = o0, hi = o1;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        const uint64_t x = from[mid];
        if (x < k || (x == k && (mine & 1)))
            lo = mid + 1;
        else
            hi = mid;
    }
    to[pair * run + (i - mine * run) + (lo - o0)] = k;
}

// 8 columns of the sum over sorted tokens i0 .. i1, in order.
template <typename T>
__device__ __forceinline__ void add_tokens(const EmbedBackward& a, int64_t i0, int64_t i1, int c, float (&s)[8]) {
    for (int64_t i = i0; i < i1; i += 4) {
        Chunk<T> k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k[j].zero();
            if (i + j < i1) load_chunk(k[j], static_cast<const T*>(a.dy.p) + (int64_t)(uint32_t)a.key0[i + j] * a.dy.ld, c, a.cols);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[8];
            k[j].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += v[e];
        }
    }
}

// Sums over pieces of kPiece sorted tokens of one id, so that a frequent id is not one workgroup's work.
template <typename T>
__global__ __launch_bounds__(256) void piece_kernel(EmbedBackward a) {
    const int64_t i0 = (int64_t)blockIdx.x * kPiece;
    const uint32_t id = (uint32_t)(a.key0[i0] >> 32);
    if ((uint32_t)(a.key0[i0 + kPiece - 1] >> 32) != id || id >= (uint64_t)a.vocab) return;
    const int c = ((int)blockIdx.y * 256 + threadIdx.x) * 8;
    if (c >= a.cols) return;
    float s[8] = {};
    add_tokens<T>(a, i0, i0 + kPiece, c, s);
    store_chunk(a.part + (int64_t)blockIdx.x * a.cols, c, a.cols, s);
}

// Number of sorted keys below `key`: 64 places are looked at at once.
__device__ __forceinline__ int64_t count_below(const uint64_t* keys, int64_t n, uint64_t key, int lane) {
    int64_t lo = 0, hi = n;  // the answer lies in lo .. hi
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step - 1;
        const int below = __popcll(__ballot(at < hi && keys[std::min(at, hi - 1)] < key));
        hi = std::min(hi, lo + (below + 1) * step - 1);
        lo += below * step;
    }
    return lo;
}

// kRows rows of the table's gradient, 2048 columns: sums of their tokens, scaled, added to the base and rounded once.
constexpr int kRows = 8;
template <typename T, typename O>
__global__ __launch_bounds__(256) void rows_kernel(EmbedBackward a) {
    const int lane = threadIdx.x & 63;
    const int64_t v0 = (int64_t)blockIdx.x * kRows;
    const int c = ((int)blockIdx.y * 256 + threadIdx.x) * 8;
    int64_t i = count_below(a.key0, a.tokens, (uint64_t)v0 << 32, lane);
    for (int64_t v = v0; v < std::min(v0 + kRows, a.vocab); ++v) {
        int64_t end = i;  // (ids of the next 64 tokens at a time)
        for (;;) {
            const bool same = end + lane < a.tokens && (int64_t)(a.key0[end + lane] >> 32) == v;
            const int n = __popcll(__ballot(same));
            end += n;
            if (n < 64) break;
        }
        const int64_t i0 = i;
        i = end;
        if (c >= a.cols) continue;
        O* const row = static_cast<O*>(a.dw) + v * a.cols;
        if (i0 == end && a.base == a.dw) continue;
        float s[8] = {};
        const int64_t p0 = (i0 + kPiece - 1) / kPiece, p1 = end / kPiece;
        if (p0 < p1) {
            add_tokens<T>(a, i0, p0 * kPiece, c, s);
            for (int64_t p = p0; p < p1; ++p) {
                Chunk<float> k;
                load_chunk(k, a.part + p * a.cols, c, a.cols);
                float v8[8];
                k.get(v8);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += v8[e];
            }
            add_tokens<T>(a, p1 * kPiece, end, c, s);
        } else {
            add_tokens<T>(a, i0, end, c, s);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] *= a.scale;
        if (a.base) {
            Chunk<O> k;
            load_chunk(k, static_cast<const O*>(a.base) + v * a.cols, c, a.cols);
            float b[8];
            k.get(b);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += b[e];
        }
        store_chunk(row, c, a.cols, s);
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
    const uint32_t slabs = (uint32_t)((a.cols + 2047) / 2048);
    if (a.tokens > 0) {
        sort_kernel<<<(uint32_t)((a.tokens + kSortRun - 1) / kSortRun), 1024, 0, st>>>(a.ids, a.tokens, a.vocab, a.key0);
        for (int64_t run = kSortRun; run < a.tokens; run *= 2) {
            merge_kernel<<<(uint32_t)((a.tokens + 255) / 256), 256, 0, st>>>(a.key0, a.key1, a.tokens, run);
            std::swap(a.key0, a.key1);
        }
        if (a.tokens >= kPiece) piece_kernel<T><<<dim3((uint32_t)(a.tokens / kPiece), slabs), 256, 0, st>>>(a);
    }
    rows_kernel<T, O><<<dim3((uint32_t)((a.vocab + kRows - 1) / kRows), slabs), 256, 0, st>>>(a);
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

EmbedPlan embed_plan(int64_t tokens, int64_t cols) {
    const auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
    EmbedPlan p = {};
    p.key1_off = up((size_t)tokens * 8);
    p.part_off = p.key1_off + (tokens > kSortRun ? up((size_t)tokens * 8) : 0);
    p.bytes = p.part_off + up((size_t)(tokens / kPiece) * cols * 4);
    return p;
}

hipError_t launch_embed_backward(int dtype, int grad_dtype, const EmbedBackward& a, hipStream_t st) {
    if (dtype == AL_DTYPE_BF16) return grad_dtype == AL_DTYPE_BF16 ? run_backward<bf16, bf16>(a, st) : run_backward<bf16, float>(a, st);
    return grad_dtype == AL_DTYPE_BF16 ? run_backward<float, bf16>(a, st) : run_backward<float, float>(a, st);
}

}  // namespace al
