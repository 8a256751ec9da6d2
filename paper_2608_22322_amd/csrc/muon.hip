// The momentum pass of the orthogonalised step: 8-bit or fp32 momentum, and the update that the products orthogonalise. Bound by memory: gradient and codes in, codes and an
// fp32 update out, 8 bytes an element with bf16 gradients (44e6 elements of a layer: 75 us, 4.7 TB/s).
#include "al_device.hpp"
#include "ortho_internal.hpp"

namespace al {

namespace {

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

typedef float f32x4 __attribute__((ext_vector_type(4)));

// The workgroup's sum, in a fixed order.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[4];
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// m <- beta m + (1 - beta) g (binary64, rounded once), its code, and the update u = m or beta m + (1 - beta) g as fp32 with its sum of squares. A
// wavefront takes blocks of 256 elements, four a lane; a workgroup kSquareUnit elements.
template <int G, bool UF>
__global__ __launch_bounds__(256) void momentum_kernel(MomentumList l, MuonArgs a, double* sums) {
    int item = 0;
    while (item + 1 < l.count && blockIdx.x >= l.begin[item + 1]) ++item;
    const MomentumItem& t = l.t[item];
    const int64_t n = t.n, unit = blockIdx.x - l.begin[item];
    const gp<const void> g = to_g(t.g);
    float* const out = t.u;
    const int lane = threadIdx.x & 63;
    const int64_t begin = unit * kSquareUnit + (threadIdx.x >> 6) * 256, end = min(n, (unit + 1) * kSquareUnit);
    double s = 0;
    for (int64_t b = begin; b < end; b += 1024) {
        const int64_t e = b + 4 * lane;
        const bool whole = e + 4 <= n;
        float gv[4] = {}, mh[4] = {};
        if (whole) {
            load_g4<G>(g, e, gv);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < n) gv[j] = grad_at_g<G>(g, e + j);
        }
        const gp<float> mf = g_as<float>(to_g(t.m));
        if constexpr (UF) {
            const double step = div127((double)to_g(t.meta)[b >> 8]);
            const uint32_t w = ld_u1<false>(g_as<const void>(g_as<const uint8_t>(to_g(t.m)) + e));
#pragma unroll
            for (int j = 0; j < 4; ++j) mh[j] = uf8_decode((int32_t)(int8_t)(uint8_t)(w >> (8 * j)), step);
        } else if (whole) {
            const float4 w = ld_f4<false>(g_as<const float>(mf) + e);
            mh[0] = w.x, mh[1] = w.y, mh[2] = w.z, mh[3] = w.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < n) mh[j] = mf[e + j];
        }
        float mn[4], uv[4];
        uint32_t top = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            mn[j] = (float)(a.beta * (double)mh[j] + a.omb * (double)gv[j]);
            uv[j] = a.nesterov ? (float)(a.beta * (double)mn[j] + a.omb * (double)gv[j]) : mn[j];
            s += (double)uv[j] * (double)uv[j];
            top = umax(top, abs_bits(mn[j]));
        }
        if constexpr (UF) {
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, m));
            const float am = u2f(top);
            // A position is x times 127 (1 / absmax), each rounded: within 2 ulps of 127 x / absmax, so that a code differs from one decided by the
            // quotient only where that lies half way between two codes (|x| half of absmax, or an absmax whose significand is a multiple of 127); other quotients of fp32 numbers are
            // 2^-33 or more away from there.
            const double r = am > 0.0f ? 127.0 * (1.0 / (double)am) : 0.0;
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = rint_low_bits((double)mn[j] * r);
            store_codes4<UF8>(g_as<uint8_t>(to_g(t.m)), e, q);
            if (lane == 0) to_g(t.meta)[b >> 8] = am;
        }
        if (whole) {
            if constexpr (!UF) st_f4<false>(mf + e, make_float4(mn[0], mn[1], mn[2], mn[3]));
            *reinterpret_cast<f32x4*>(out + e) = f32x4{uv[0], uv[1], uv[2], uv[3]};
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (e + j >= n) continue;
                if constexpr (!UF) mf[e + j] = mn[j];
                out[e + j] = uv[j];
            }
        }
    }
    s = block_sum(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

}  // namespace

hipError_t launch_momentum(const MuonArgs& a, const MomentumList& l, double* sums, hipStream_t s) {
    const uint32_t grid = l.begin[l.count];
    if (a.grad_bf16) {
        if (a.uf8) momentum_kernel<G_BF16, true><<<grid, 256, 0, s>>>(l, a, sums);
        else momentum_kernel<G_BF16, false><<<grid, 256, 0, s>>>(l, a, sums);
    } else {
        if (a.uf8) momentum_kernel<G_F32, true><<<grid, 256, 0, s>>>(l, a, sums);
        else momentum_kernel<G_F32, false><<<grid, 256, 0, s>>>(l, a, sums);
    }
    return hipGetLastError();
}

}  // namespace al
