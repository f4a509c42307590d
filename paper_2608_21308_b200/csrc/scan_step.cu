// Gated linear recurrence, recurrent form: a few tokens of every sequence on its state (decoding).  A thread has two channels; the state is read once and
// written once.  A call is launch latency up to many sequences (64 of 2048 channels: 2 MB).
#include "scan_common.cuh"

namespace e2ttt {
namespace {
using namespace scan;

constexpr int kStepThreads = 64;  // 16 CTAs for 2048 channels

template <typename IO, bool GATE, bool UNIT> __global__ void __launch_bounds__(kStepThreads) scan_step_kernel(const ScanArgs a, const bool pair, const int groups) {
    const int b = blockIdx.x / groups, c0 = ((blockIdx.x - b * groups) * kStepThreads + threadIdx.x) * 2, D = a.s.D;
    const int n = min(2, D - c0);
    if (n <= 0) return;
    const bool even = (D & 1) == 0 && ((reinterpret_cast<uintptr_t>(a.rate) | reinterpret_cast<uintptr_t>(a.h_init) | reinterpret_cast<uintptr_t>(a.h_final)) & 7) == 0;
    const Pairs pairs = make_pairs();
    float2 rate = load2<float>(a.rate, c0, n, even);
    rate = make_float2(-rate.x, -rate.y);
    float2 h = load2<float>(a.h_init, (int64_t)b * D + c0, n, even);
    for (int t = 0; t < a.s.L; ++t) {
        const int64_t at = ((int64_t)b * a.s.L + t) * D + c0;
        float2 u = load2<IO>(a.x, at, n, pair);
        const float2 r = load2<IO>(a.r, at, n, pair);
        if (GATE) u = mul2(u, sigmoid2<IO>(pairs, capped(load2<IO>(a.g, at, n, pair))));
        const Decay d = decay<IO, UNIT, false>(pairs, sigmoid2<IO>(pairs, capped(r)), rate);
        if (a.starts && a.starts[(int64_t)b * a.s.L + t]) {
            h = u;
        } else {
            if (UNIT) u = mul2(u, sqrt_minus(d.minus));
            h = add2(fade<false>(h, d.c, d.far), u);
        }
        store2<IO>(a.h, at, n, pair, h);
    }
    store2<float>(a.h_final, (int64_t)b * D + c0, n, even, h);
}

template <typename IO, bool GATE> int launch(const ScanArgs& a, bool pair, cudaStream_t st) {
    const int groups = (a.s.D + 2 * kStepThreads - 1) / (2 * kStepThreads);
    const unsigned grid = (unsigned)(a.s.B * (int64_t)groups);
    if (a.s.unit) scan_step_kernel<IO, GATE, true><<<grid, kStepThreads, 0, st>>>(a, pair, groups);
    else scan_step_kernel<IO, GATE, false><<<grid, kStepThreads, 0, st>>>(a, pair, groups);
    return (int)cudaGetLastError();
}

}  // namespace

int scan_step_launch(const ScanArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.r) | reinterpret_cast<uintptr_t>(a.g) | reinterpret_cast<uintptr_t>(a.h);
    const bool pair = a.s.D % 2 == 0 && all % (a.s.f32 ? 8 : 4) == 0;
    if (a.s.f32) return a.s.gate ? launch<float, true>(a, pair, st) : launch<float, false>(a, pair, st);
    return a.s.gate ? launch<__nv_bfloat16, true>(a, pair, st) : launch<__nv_bfloat16, false>(a, pair, st);
}

}  // namespace e2ttt
