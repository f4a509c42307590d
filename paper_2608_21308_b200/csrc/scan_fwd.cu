// Gated linear recurrence, forward.  h_t = a_t h_{t-1} + b_t is linear in the state: over a run of tokens h_out = P h_in + h', P the product of the a_t and h' the run's
// end from a zero state.  A CTA has 64 channels of a sequence and walks its tokens 64 at a time; a lane has two channels, a warp eight tokens of the tile, whose
// P and h' meet in shared memory.
#include "pack8.cuh"
#include "scan_common.cuh"

namespace e2ttt {
namespace {
using namespace scan;

constexpr int kTok = 8;  // tokens of a thread in a tile

template <typename IO, bool GATE, bool UNIT, bool PACK>
__global__ void __launch_bounds__(kThreads) scan_fwd_kernel(const ScanArgs a, const bool pair) {
    __shared__ float4 runs[2][kWarps][32];
    const int D = a.s.D, L = a.s.L, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t blocks = a.s.blocks(), spans = a.s.spans();
    const int64_t b = blockIdx.x / blocks, blk = blockIdx.x - b * blocks;
    const int c0 = (int)blk * kScanCh + 2 * lane, n = max(0, min(2, D - c0));
    float2 rate = load2<float>(a.rate, c0, n, false);
    rate = make_float2(-rate.x, -rate.y);
    float2 carry = a.h_init ? load2<float>(a.h_init, b * D + c0, n, false) : dup(0.0f);
    int flip = 0;
    for (int64_t tile = 0; tile < spans; ++tile, flip ^= 1) {
        const int t0 = (int)(tile * kScanSpan) + warp * kTok;
        if (a.states && warp == 0) store2<float>(a.states, (b * spans + tile) * D + c0, n, false, carry);
        float2 h[kTok], P[kTok], hh = dup(0.0f), pp = dup(1.0f);
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            const int t = t0 + j;
            const bool in = t < L;
            const int64_t at = (b * L + t) * D + c0;
            const float2 x = load2<IO>(a.x, at, in ? n : 0, pair), r = load2<IO>(a.r, at, in ? n : 0, pair);
            const float2 g = GATE ? load2<IO>(a.g, at, in ? n : 0, pair) : dup(0.0f);
            if (PACK) {
                const float2 v[3] = {x, r, g};
#pragma unroll
                for (int k = 0; k < (GATE ? 3 : 2); ++k) {
                    uint32_t m = max(pack8::magnitude(v[k].x), pack8::magnitude(v[k].y));
#pragma unroll
                    for (int s = 1; s < 16; s <<= 1) m = max(m, __shfl_xor_sync(kAll, m, s));
                    const uint32_t byte = pack8::scale_byte(m);
                    const float w[2] = {v[k].x, v[k].y};
                    const int64_t row = (b * blocks + blk) * spans * kScanSpan + t;
                    *reinterpret_cast<pack8::Codes<2>*>(a.codes + k * a.code_step + row * kScanCh + 2 * lane) = pack8::encode<2>(w, byte);
                    if ((lane & 15) == 0) a.scales[k * a.scale_step + row * 2 + (lane >> 4)] = (uint8_t)byte;
                }
            }
            float2 u = x;
            if (GATE) u = mul2(u, sigmoid2<IO>(g));
            const Decay d = decay<IO, UNIT, false>(sigmoid2<IO>(r), rate);
            if (in && a.starts && a.starts[b * L + t]) {
                hh = u;
                pp = dup(0.0f);
            } else if (in) {
                if (UNIT) u = mul2(u, mul2(d.one, inv_sqrt2<IO>(d.one)));
                hh = add2(fade<false>(hh, d.c, d.far), u);
                pp = fade<false>(pp, d.c, d.far);
            }
            h[j] = hh;
            P[j] = pp;
        }
        runs[flip][warp][lane] = make_float4(pp.x, pp.y, hh.x, hh.y);
        __syncthreads();
        float2 in = carry;
        for (int w = 0; w < kWarps; ++w) {
            const float4 q = runs[flip][w][lane];
            if (w == warp) in = carry;
            carry.x = q.x == 0.0f ? q.z : fmaf(q.x, carry.x, q.z);
            carry.y = q.y == 0.0f ? q.w : fmaf(q.y, carry.y, q.w);
        }
        if (a.h) {
#pragma unroll
            for (int j = 0; j < kTok; ++j) {
                if (t0 + j >= L) continue;
                float2 y;
                y.x = P[j].x == 0.0f ? h[j].x : fmaf(P[j].x, in.x, h[j].x);
                y.y = P[j].y == 0.0f ? h[j].y : fmaf(P[j].y, in.y, h[j].y);
                store2<IO>(a.h, (b * L + t0 + j) * D + c0, n, pair, y);
            }
        }
    }
    if (a.h_final && warp == 0) store2<float>(a.h_final, b * D + c0, n, false, carry);
}

template <typename IO, bool GATE, bool UNIT> int launch(const ScanArgs& a, bool pair, cudaStream_t st) {
    const unsigned grid = (unsigned)(a.s.B * a.s.blocks());
    if (a.codes) scan_fwd_kernel<IO, GATE, UNIT, true><<<grid, kThreads, 0, st>>>(a, pair);
    else scan_fwd_kernel<IO, GATE, UNIT, false><<<grid, kThreads, 0, st>>>(a, pair);
    return (int)cudaGetLastError();
}
template <typename IO> int dispatch(const ScanArgs& a, bool pair, cudaStream_t st) {
    if (a.s.gate) return a.s.unit ? launch<IO, true, true>(a, pair, st) : launch<IO, true, false>(a, pair, st);
    return a.s.unit ? launch<IO, false, true>(a, pair, st) : launch<IO, false, false>(a, pair, st);
}

}  // namespace

int scan_parts(const ScanShape&) { return 1; }

int scan_fwd_launch(const ScanArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.r) | reinterpret_cast<uintptr_t>(a.g) | reinterpret_cast<uintptr_t>(a.h);
    const bool pair = a.s.D % 2 == 0 && all % (a.s.f32 ? 8 : 4) == 0;
    return a.s.f32 ? dispatch<float>(a, pair, st) : dispatch<__nv_bfloat16>(a, pair, st);
}

}  // namespace e2ttt
