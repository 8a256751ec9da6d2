// Softmax cross entropy of a linear head, logits = h w^T, without keeping the logits.
//
//   loss[t] = lse[t] - logit[t][target],  lse[t] = log sum exp logits[t]
//   d[t][v] = coef[t] (exp(logit[t][v] - lse[t]) - [v = target]),  dh = d w,  dw = d^T h + base
//
// The statistics come from the end of the product itself: a wavefront reduces its 64 (32) columns of each row to a maximum and a sum, and a pass over
// those gives the row's. lse is kept as these two numbers, lse = top + log(sum): rounded to one, it would be off by 2^-24 of the logits' size, which for a confident token is more than its loss
// and is the same factor in all of a row's probabilities. For the gradients the product is taken once more, a piece of the vocabulary at a time, whose end forms d in bf16 (one
// part, or two where a gradient is wanted in fp32); two more products use it while it is in the caches. A fourth product for three, but no
// tokens x vocabulary matrix: what is kept is tokens x piece.
//
// Bound by the matrix cores (8192 tokens, 32000 x 2048, bf16 gradients: 3.68 ms, the four products at 1.0 to 1.2 PFLOP/s), for one token by reading w (32000 x 4096: 54 us, the
// product 6.5 TB/s), for fp32 gradients by the ends that read a base and write dw between rounds of tiles (1501 tokens, 32003 x 1750: 1.16 ms).
#include <algorithm>
#include <cmath>

#include "mm_device.hpp"
#include "vocab_internal.hpp"

namespace al {

namespace {

__device__ __forceinline__ int64_t target_at(const Ids& ids, int64_t t) {
    return ids.wide ? static_cast<const int64_t*>(ids.p)[t] : (int64_t) static_cast<const int32_t*>(ids.p)[t];
}

// Rows of h padded with zeros to tp x dp; those without a target are zero (what stands there, NaN too, must not reach dw). w alike, every row kept.
__global__ __launch_bounds__(256) void pad_kernel(Mat x, int64_t rows, int32_t cols, int64_t rp, int32_t cp, Ids target, int64_t vocab, uint16_t* out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int chunks = cp / 8;
    const int64_t r = i / chunks;
    const int c = (int)(i - r * chunks) * 8;
    if (r >= rp) return;
    Chunk<bf16> k;
    k.zero();
    bool keep = r < rows;
    if (keep && target.p) {
        const int64_t t = target_at(target, r);
        keep = t >= 0 && t < vocab;
    }
    if (keep) load_chunk(k, static_cast<const bf16*>(x.p) + r * x.ld, c, cols);
    *reinterpret_cast<u32x4*>(out + r * cp + c) = k.q;
}

constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

struct Stat {
    float top, sum;  // largest logit of some columns, and the sum of exp(logit - top)
};
struct Norm {
    float top, log2;  // of a row: the largest logit, and the logarithm of the sum of exp(logit - top) to base 2
};

// End of the statistics' product: a wavefront's columns of a row as one Stat, and the target's logit where it is among them.
struct EndStats {
    static constexpr bool kRows = true;
    Stat* stats;    // [token of the block][group]
    float* at;      // the target's logit
    Ids target;
    int64_t t0;     // first token of the block
    int32_t tokens, vocab, groups;
    template <int FM, int FN>
    __device__ __forceinline__ void rows(int m, int n, int lane, const f32x4 (&v)[FM][FN]) const {
        int64_t y[FM];
#pragma unroll
        for (int i = 0; i < FM; ++i) y[i] = m + 16 * i < tokens ? target_at(target, t0 + m + 16 * i) - n : -1;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            row<FN>(m + 16 * i, n, lane, v[i], y[i]);
        }
    }
    template <int FN>
    __device__ __forceinline__ void row(int m, int n, int lane, const f32x4 (&v)[FN], int64_t y) const {
        float top = -__builtin_inff(), sum = 0;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + 16 * j + r < vocab) top = fmaxf(top, v[j][r]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + 16 * j + r < vocab) sum += exp_of(v[j][r] - from);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (m >= tokens) return;
        if (lane < 16) {
            const int g = (n - 4 * (lane >> 4)) / (16 * FN);
            if (g < groups) stats[(int64_t)m * groups + g] = {top, sum};
        }
        if (y >= 0 && y < 16 * FN && (y & 12) == 0) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (y == 16 * j + r && n + 16 * j + r < vocab) at[m] = v[j][r];
        }
    }
};

// What a row is normed by, its loss and the gradients' coefficient of each token; tokens behind the last have coefficient 0.
__global__ __launch_bounds__(256) void loss_kernel(const Stat* stats, const float* at, int32_t groups, int64_t t0, int32_t tokens, int32_t tokens_padded, int64_t vocab,
                                                   Ids target, const float* weight, float scale, float* loss, float* lse, Norm* norms, float* coef) {
    const int lane = threadIdx.x & 63, m = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= tokens_padded) return;
    if (m >= tokens) {
        if (lane == 0 && coef) {
            norms[t0 + m] = {0.0f, 0.0f};
            coef[t0 + m] = 0.0f;
        }
        return;
    }
    float top = -__builtin_inff(), sum = 0;
    const Stat* const s = stats + (int64_t)m * groups;
    bool bad = false;
    for (int g = lane; g < groups; g += 512) {
        Stat x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = g + 64 * j < groups ? s[g + 64 * j] : Stat{-__builtin_inff(), 0.0f};
        float t = top;
#pragma unroll
        for (int j = 0; j < 8; ++j) t = fmaxf(t, x[j].top);
        if (t != -__builtin_inff()) {
            sum *= exp_of(top - t);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += x[j].sum * exp_of(x[j].top - t);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) bad |= x[j].sum != x[j].sum;
        top = t;
    }
    for (int k = 1; k < 64; k <<= 1) {
        const float ot = __shfl_xor(top, k), os = __shfl_xor(sum, k), t = fmaxf(top, ot);
        if (t != -__builtin_inff()) sum = sum * exp_of(top - t) + os * exp_of(ot - t);
        top = t;
    }
    bad = __any(bad);
    if (lane) return;
    const float l = bad ? __builtin_nanf("") : logf(sum);
    const int64_t y = target_at(target, t0 + m);
    const bool has = y >= 0 && y < vocab;
    if (loss) loss[t0 + m] = has ? (top - at[m]) + l : 0.0f;
    if (lse) lse[t0 + m] = has ? top + l : 0.0f;
    if (coef) {
        norms[t0 + m] = {top, l * kLog2e};
        coef[t0 + m] = has ? scale * (weight ? weight[t0 + m] : 1.0f) : 0.0f;
    }
}

// End of a piece's product: d in bf16 parts, zeros past the last token and the last column.
struct EndGrad {
    static constexpr bool kRows = true;
    uint16_t* d;
    int64_t size;  // from the high part to the low
    int32_t ld, parts, tokens_padded;
    const Norm* norms;
    const float* coef;
    Ids target;
    int64_t v0;
    int32_t tokens, columns;
    // (what belongs to the rows is loaded at once, before any of them is written: one after the other 8192 x 8192 logits of K = 2048 take 285 us, so 266)
    template <int FM, int FN>
    __device__ __forceinline__ void rows(int m, int n, int lane, const f32x4 (&v)[FM][FN]) const {
        float c[FM];
        Norm l[FM];
        int64_t y[FM];
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int r = min(m + 16 * i, tokens_padded - 1);
            c[i] = coef[r];
            l[i] = norms[r];
            y[i] = r < tokens ? target_at(target, r) - v0 - n : -1;
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) quad(m + 16 * i, n + 16 * j, v[i][j], c[i], l[i], y[i] - 16 * j);
        }
    }
    __device__ __forceinline__ void quad(int m, int n, f32x4 v, float c, Norm l, int64_t y) const {
        if (m >= tokens_padded || n >= ld) return;
        f32x4 g;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[r] - l.top, kLog2e, -l.log2)) - (y == r ? 1.0f : 0.0f);
            g[r] = c != 0.0f && n + r < columns ? c * p : 0.0f;
        }
        uint16_t* const q = d + (int64_t)m * ld + n;
        const u32x2 hi = {pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3])};
        *reinterpret_cast<u32x2*>(q) = hi;
        if (parts > 1) {
            const float h[4] = {bits_f(hi[0] << 16), bits_f(hi[0] & 0xffff0000u), bits_f(hi[1] << 16), bits_f(hi[1] & 0xffff0000u)};
            *reinterpret_cast<u32x2*>(q + size) = u32x2{pack_bf16(g[0] - h[0], g[1] - h[1]), pack_bf16(g[2] - h[2], g[3] - h[3])};
        }
    }
};

template <typename O>
__device__ __forceinline__ f32x4 get4(const O* p, int in) {
    f32x4 v = {};
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (r < in) v[r] = to_f(p[r]);
    return v;
}
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ f32x4 load4(const bf16* p, int in) {
    if (in < 4) return get4(p, in);
    const u32x2 b = *reinterpret_cast<const u32x2_a2*>(p);
    return f32x4{bits_f(b[0] << 16), bits_f(b[0] & 0xffff0000u), bits_f(b[1] << 16), bits_f(b[1] & 0xffff0000u)};
}
__device__ __forceinline__ f32x4 load4(const float* p, int in) {
    if (in < 4) return get4(p, in);
    return *reinterpret_cast<const f32x4_a4*>(p);
}
__device__ __forceinline__ void save4(bf16* p, int in, f32x4 v) {
    if (in >= 4) {
        *reinterpret_cast<u32x2_a2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int r = 0; r < 3; ++r)
        if (r < in) put(p + r, v[r]);
}
__device__ __forceinline__ void save4(float* p, int in, f32x4 v) {
    if (in >= 4) {
        *reinterpret_cast<f32x4_a4*>(p) = v;
        return;
    }
#pragma unroll
    for (int r = 0; r < 3; ++r)
        if (r < in) p[r] = v[r];
}

// End of dw's and dh's products: rows x cols of `out` (bf16 or fp32), to which `base` (the same type) and `sum` (fp32, packed) are added where they are
// not NULL. An intermediate dh goes to `sum` itself.
struct EndSum {
    void* out;
    const void* base;
    const float* sum;
    int64_t ld, sum_ld;
    int32_t rows, cols, out_bf16;
    __device__ __forceinline__ void operator()(int m, int n, f32x4 v) const {
        if (m >= rows || n >= cols) return;
        const int in = min(4, cols - n);
        const int64_t i = m * ld + n;
        if (sum) v += load4(sum + m * sum_ld + n, in);
        if (out_bf16) {
            if (base) v += load4(static_cast<const bf16*>(base) + i, in);
            save4(static_cast<bf16*>(out) + i, in, v);
        } else {
            if (base) v += load4(static_cast<const float*>(base) + i, in);
            save4(static_cast<float*>(out) + i, in, v);
        }
    }
};

// PA: parts of A.
template <bool AK, bool BK, int ENDS, int PA, class E>
hipError_t product(const MmCut& cut, Mm p, const E& end, hipStream_t st) {
    p.splits = cut.splits;
    p.segs = mm_segments(cut.tile, 1 + PA);
    p.amask = p.segs > 1 ? 2u : 0u;
    if (cut.tile == 256) return mm_launch<bf16, 256, AK, BK, ENDS, 1>(p, end, st);
    if (cut.tile == 128) return mm_launch<bf16, 128, AK, BK, ENDS, 1>(p, end, st);
    return mm_launch<bf16, 64, AK, BK, ENDS, PA>(p, end, st);
}

void pad(Mat x, int64_t rows, int32_t cols, int64_t rp, int32_t cp, Ids target, int64_t vocab, uint16_t* out, hipStream_t st) {
    pad_kernel<<<(uint32_t)((rp * (cp / 8) + 255) / 256), 256, 0, st>>>(x, rows, cols, rp, cp, target, vocab, out);
}

int wave_columns(int tile) { return tile == 64 ? 32 : 64; }

}  // namespace

XentPlan xent_plan(int64_t tokens, int64_t hidden, int64_t vocab, int64_t ldw, int dh_dtype, int grad_dtype, bool dh, bool dw) {
    XentPlan p = {};
    p.tokens = tokens;
    p.hidden = hidden;
    p.vocab = vocab;
    p.tp = (int32_t)((tokens + 63) / 64 * 64);
    p.dp = (int32_t)((hidden + 63) / 64 * 64);
    p.pack = hidden % 8 != 0 || ldw % 8 != 0 || ldw >= (1 << 23);
    p.block = (int32_t)std::min<int64_t>(p.tp, 16384);
    p.dh_parts = dh ? (dh_dtype == AL_DTYPE_F32 ? 2 : 1) : 0;
    p.dw_parts = dw ? (grad_dtype == AL_DTYPE_F32 ? 2 : 1) : 0;
    p.parts = std::max(p.dh_parts, p.dw_parts);
    const int64_t turns = p.dp / kMmTurn;
    // (16384 tokens of up to 64 features by 2^24 columns are 2^32 threads of 128-wide tiles: two passes)
    for (;; p.block = (p.block / 2 + 63) / 64 * 64) {
        p.logits = mm_cut(p.block, vocab, turns, 2);
        p.logits.splits = 1;
        if (mm_threads(p.logits, p.block, vocab) < (int64_t(1) << 32)) break;
    }
    const auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
    size_t off = 0;
    const auto take = [&](size_t bytes) {
        const size_t at = off;
        off += up(bytes);
        return at;
    };
    p.h_off = take((size_t)p.tp * p.dp * 2);
    p.w_off = take(p.pack ? (size_t)vocab * p.dp * 2 : 0);
    p.groups = (int32_t)((vocab + wave_columns(p.logits.tile) - 1) / wave_columns(p.logits.tile));
    p.stat_off = take((size_t)p.block * p.groups * sizeof(Stat) + (size_t)p.block * 4);
    if (p.parts) {
        const int64_t room = (int64_t(1) << 26) / p.tp / 256 * 256;
        p.piece = (int32_t)std::min<int64_t>((vocab + 63) / 64 * 64, std::max<int64_t>(256, room));
        p.back = mm_cut(p.tp, p.piece, turns, 2);
        p.back.splits = 1;
        p.dh = mm_cut(p.tp, hidden, p.piece / kMmTurn, 1 + std::max(1, p.dh_parts));
        p.dw = mm_cut(p.piece, hidden, p.tp / kMmTurn, 1 + std::max(1, p.dw_parts));
        p.norm_off = take((size_t)p.tp * sizeof(Norm));
        p.coef_off = take((size_t)p.tp * 4);
        p.d_off = take((size_t)p.tp * p.piece * 2 * p.parts);
        p.dh_off = take(dh && p.piece < vocab ? (size_t)p.tp * hidden * 4 : 0);
        p.part_off = take(std::max(dh ? mm_part_bytes(p.dh, p.tp, hidden) : 0, dw ? mm_part_bytes(p.dw, p.piece, hidden) : 0));
    }
    p.bytes = off;
    return p;
}

hipError_t launch_xent(const XentPlan& p, const Xent& a, void* ws, hipStream_t st) {
    char* const base = static_cast<char*>(ws);
    uint16_t* const h = reinterpret_cast<uint16_t*>(base + p.h_off);
    // Without dw, rows without a target or past the last do no harm, and whole turns of aligned rows are read where they are (one token, 32000 x 4096: 47 and 4 us for 42).
    const bool as_is = p.dw_parts == 0 && p.hidden == p.dp && a.h.ld % 8 == 0 && a.h.ld < (1 << 23) && (reinterpret_cast<uintptr_t>(a.h.p) & 15u) == 0;
    if (!as_is) pad(a.h, p.tokens, (int32_t)p.hidden, p.tp, p.dp, a.target, p.vocab, h, st);
    MmOperand w = {static_cast<const uint16_t*>(a.w.p), 0, (int32_t)a.w.ld, (int32_t)p.vocab, (int32_t)p.hidden};
    if (p.pack) {
        uint16_t* const to = reinterpret_cast<uint16_t*>(base + p.w_off);
        pad(a.w, p.vocab, (int32_t)p.hidden, p.vocab, p.dp, Ids{nullptr, 0}, p.vocab, to, st);
        w.p = to;
        w.ld = w.cols = p.dp;
    }
    MmOperand oh = {h, 0, p.dp, p.tp, p.dp};
    if (as_is) oh = {static_cast<const uint16_t*>(a.h.p), 0, (int32_t)a.h.ld, (int32_t)p.tokens, p.dp};
    Stat* const stats = reinterpret_cast<Stat*>(base + p.stat_off);
    Norm* const norms = p.parts ? reinterpret_cast<Norm*>(base + p.norm_off) : nullptr;
    float* const coef = p.parts ? reinterpret_cast<float*>(base + p.coef_off) : nullptr;
    // The logits' products. (Rows of w that end with a whole turn could take kMmWhole. Its addresses wait in registers, kMmLast's are formed beside the products: 8192 x 32000 x 2048 935 us
    // so, 953 with the former; kMmZeros' choice for each piece makes both products about 1% longer.)
    const auto logits = [&](const MmCut& cut, const Mm& g, const auto& end) {
        return w.cols < p.dp ? product<true, true, kMmZeros, 1>(cut, g, end, st) : product<true, true, kMmLast, 1>(cut, g, end, st);
    };
    Mm q = {};
    q.part = reinterpret_cast<float*>(base + p.part_off);
    hipError_t e;
    float* const at = reinterpret_cast<float*>(stats + (size_t)p.block * p.groups);
    for (int64_t t0 = 0; t0 < p.tokens; t0 += p.block) {
        const int32_t padded = (int32_t)std::min<int64_t>(p.block, p.tp - t0), n = (int32_t)std::min<int64_t>(p.block, p.tokens - t0);
        Mm g = q;
        g.a = oh;
        g.a.p += t0 * oh.ld;
        g.a.rows = (int32_t)std::min<int64_t>(padded, oh.rows - t0);
        g.b = w;
        g.m = n;
        g.n = (int32_t)p.vocab;
        g.turns = p.dp / kMmTurn;
        const EndStats end = {stats, at, a.target, t0, n, (int32_t)p.vocab, p.groups};
        if ((e = logits(p.logits, g, end)) != hipSuccess) return e;
        loss_kernel<<<(uint32_t)((padded + 3) / 4), 256, 0, st>>>(stats, at, p.groups, t0, n, padded, p.vocab, a.target, a.weight, a.scale, a.loss, a.lse, norms, coef);
    }
    if (!p.parts) return hipGetLastError();
    uint16_t* const d = reinterpret_cast<uint16_t*>(base + p.d_off);
    float* const sum = reinterpret_cast<float*>(base + p.dh_off);
    for (int64_t v0 = 0; v0 < p.vocab; v0 += p.piece) {
        const int32_t n = (int32_t)std::min<int64_t>(p.piece, p.vocab - v0), np = (n + 63) / 64 * 64;
        const bool first = v0 == 0, last = v0 + p.piece >= p.vocab;
        const int64_t size = (int64_t)p.tp * np;
        MmOperand wp = w;
        wp.p += v0 * w.ld;
        wp.rows = n;
        Mm g = q;
        g.a = oh;
        g.b = wp;
        g.m = p.tp;
        g.n = np;
        g.turns = p.dp / kMmTurn;
        const EndGrad end = {d, size, np, p.parts, p.tp, norms, coef, a.target, v0, (int32_t)p.tokens, n};
        if ((e = logits(p.back, g, end)) != hipSuccess) return e;
        const MmOperand od = {d, size, np, p.tp, np};
        if (p.dh_parts) {
            Mm g2 = q;
            g2.a = od;
            g2.b = wp;
            g2.m = p.tp;
            g2.n = (int32_t)p.hidden;
            g2.turns = np / kMmTurn;
            EndSum s = {};
            s.sum = first ? nullptr : sum;
            s.sum_ld = p.hidden;
            s.cols = (int32_t)p.hidden;
            if (last) {
                s.out = a.dh.p;
                s.ld = a.dh.ld;
                s.rows = (int32_t)p.tokens;
                s.out_bf16 = a.dh_bf16;
            } else {
                s.out = sum;
                s.ld = p.hidden;
                s.rows = p.tp;
            }
            e = p.dh_parts > 1 ? product<true, false, kMmLast, 2>(p.dh, g2, s, st) : product<true, false, kMmLast, 1>(p.dh, g2, s, st);
            if (e != hipSuccess) return e;
        }
        if (p.dw_parts) {
            Mm g3 = q;
            g3.a = od;
            g3.b = oh;
            g3.m = n;
            g3.n = (int32_t)p.hidden;
            g3.turns = p.tp / kMmTurn;
            EndSum s = {};
            const int64_t skip = v0 * p.hidden * (a.dw_bf16 ? 2 : 4);
            s.out = static_cast<char*>(a.dw) + skip;
            s.base = a.base ? static_cast<const char*>(a.base) + skip : nullptr;
            s.ld = p.hidden;
            s.rows = n;
            s.cols = (int32_t)p.hidden;
            s.out_bf16 = a.dw_bf16;
            e = p.dw_parts > 1 ? product<false, false, kMmWhole, 2>(p.dw, g3, s, st) : product<false, false, kMmWhole, 1>(p.dw, g3, s, st);
            if (e != hipSuccess) return e;
        }
    }
    return hipGetLastError();
}

}  // namespace al
