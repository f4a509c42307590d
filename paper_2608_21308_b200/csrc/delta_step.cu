// Gated delta rule, recurrent form: a few tokens of every sequence on its state (decoding).  One pass over the state, read and
// written once whatever the number of tokens: 8 bytes a state value against 6 flop a value and token, so HBM bounds a call of many sequences
// and latency a call of few.  Eight lanes hold a state row (16-byte pieces, 128 bytes of a row per load), a warp eight rows: 4 KB in
// flight per warp before the first product, and three shuffles end a row's sums.  fp32 arithmetic, nothing rounded but o.
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

constexpr int kRows = 2;      // rows per group of eight lanes
constexpr int kThreads = 64;  // 16 rows per CTA: 16 heads of 128 rows are 128 CTAs

__device__ __forceinline__ float sum8(float x) {
    x += __shfl_xor_sync(kAll, x, 1);
    x += __shfl_xor_sync(kAll, x, 2);
    return x + __shfl_xor_sync(kAll, x, 4);
}

template <typename IO, bool VEC> __device__ __forceinline__ void ld4(const IO* p, int c, int d, float (&x)[4]) {
    if (VEC) {  // d is a multiple of 4 and so is c
        if (c < d) {
            if (sizeof(IO) == 2) {
                const uint2 raw = *reinterpret_cast<const uint2*>(p + c);
                x[0] = __uint_as_float(raw.x << 16); x[1] = __uint_as_float(raw.x & 0xffff0000u);
                x[2] = __uint_as_float(raw.y << 16); x[3] = __uint_as_float(raw.y & 0xffff0000u);
            } else {
                const float4 y = *reinterpret_cast<const float4*>(p + c);
                x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
            }
        } else {
            x[0] = x[1] = x[2] = x[3] = 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = c + j < d ? to_f32(p[c + j]) : 0.0f;
    }
}

template <typename IO, int NI, bool VEC>
__global__ void __launch_bounds__(kThreads) delta_step_kernel(const DeltaStepArgs a) {
    const DeltaShape& s = a.s;
    const int lane = threadIdx.x & 31, l8 = lane & 7;
    constexpr int per = kThreads / 8 * kRows;
    const int groups = (s.dv + per - 1) / per;
    const int64_t n = blockIdx.x / groups, nk = (n / s.H) * s.Hk + (n % s.H) / (s.H / s.Hk);
    const int row = (int)(blockIdx.x % groups) * per + (int)(threadIdx.x >> 3) * kRows;
    float S[kRows][NI][4];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const float* p = a.S + ((size_t)n * s.dv + row + r) * s.dk;
#pragma unroll
        for (int i = 0; i < NI; ++i) ld4<float, VEC>(p, i * 32 + l8 * 4, row + r < s.dv ? s.dk : 0, S[r][i]);
    }
    const IO* qp = reinterpret_cast<const IO*>(a.q) + (size_t)nk * s.L * s.dk;
    const IO* kp = reinterpret_cast<const IO*>(a.k) + (size_t)nk * s.L * s.dk;
    const IO* vp = reinterpret_cast<const IO*>(a.v) + (size_t)n * s.L * s.dv;
    IO* op = reinterpret_cast<IO*>(a.o) + (size_t)n * s.L * s.dv;
    for (int t = 0; t < s.L; ++t) {
        float k[NI][4], q[NI][4], v[kRows];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            ld4<IO, VEC>(kp + (size_t)t * s.dk, i * 32 + l8 * 4, s.dk, k[i]);
            ld4<IO, VEC>(qp + (size_t)t * s.dk, i * 32 + l8 * 4, s.dk, q[i]);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) v[r] = row + r < s.dv ? to_f32(vp[(size_t)t * s.dv + row + r]) : 0.0f;
        const float gamma = expf(a.log_gamma[(size_t)n * s.L + t]), eta = a.eta[(size_t)n * s.L + t];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float sk[2] = {0.0f, 0.0f}, so[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    S[r][i][j] *= gamma;
                    sk[j & 1] = fmaf(S[r][i][j], k[i][j], sk[j & 1]);
                }
            const float u = eta * (v[r] - sum8(sk[0] + sk[1]));
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    S[r][i][j] = fmaf(u, k[i][j], S[r][i][j]);
                    so[j & 1] = fmaf(S[r][i][j], q[i][j], so[j & 1]);
                }
            const float o = s.scale * sum8(so[0] + so[1]);
            if (l8 == 0 && row + r < s.dv) op[(size_t)t * s.dv + row + r] = from_f32<IO>(o);
        }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (row + r >= s.dv) continue;
        float* p = a.S_out + ((size_t)n * s.dv + row + r) * s.dk;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int c = i * 32 + l8 * 4;
            if (VEC) {
                if (c < s.dk) *reinterpret_cast<float4*>(p + c) = make_float4(S[r][i][0], S[r][i][1], S[r][i][2], S[r][i][3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < s.dk) p[c + j] = S[r][i][j];
            }
        }
    }
}

template <typename IO> int launch(const DeltaStepArgs& a, cudaStream_t st) {
    const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    const bool vec = a.s.dk % 4 == 0 && (at(a.S) | at(a.S_out)) % 16 == 0 && (at(a.q) | at(a.k)) % (4 * sizeof(IO)) == 0;
    constexpr int per = kThreads / 8 * kRows;
    const unsigned grid = (unsigned)((int64_t)a.s.B * a.s.H * ((a.s.dv + per - 1) / per));
    if (a.s.dk <= 64) {
        if (vec) delta_step_kernel<IO, 2, true><<<grid, kThreads, 0, st>>>(a);
        else delta_step_kernel<IO, 2, false><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (vec) delta_step_kernel<IO, 4, true><<<grid, kThreads, 0, st>>>(a);
        else delta_step_kernel<IO, 4, false><<<grid, kThreads, 0, st>>>(a);
    }
    return (int)cudaGetLastError();
}

}  // namespace

int delta_step_launch(const DeltaStepArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return a.s.f32 ? launch<float>(a, st) : launch<__nv_bfloat16>(a, st);
}

}  // namespace e2ttt
