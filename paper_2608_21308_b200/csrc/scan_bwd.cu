// Gated linear recurrence, reverse pass.  The adjoint of h runs backwards by the same rule: lam_t = d_h_t + a_{t+1} lam_{t+1}.  A tile of 64 tokens starts from its saved
// state and from the adjoint that the tokens after it hand on; a warp has eight of its tokens.  Per run of tokens P (the product of the a_t), the end h' of the states from
// zero and the adjoint handed on from zero meet in shared memory, once for both directions.  With a, i, s the gates and u = i x:
//   d_x = lam s i,   d_a_in = lam s u (1 - i),   d_log_a = a lam (h_{t-1} - a u / s),   d_a_decay = d_log_a log_a (1 - sg),   d_rate = -sum d_log_a sg.
#include "pack8.cuh"
#include "scan_common.cuh"

namespace e2ttt {
namespace {
using namespace scan;

constexpr int kTok = 8;

template <typename IO, bool GATE, bool UNIT, bool PACK>
__global__ void __launch_bounds__(kThreads) scan_bwd_kernel(const ScanBwdArgs ba, const bool pair) {
    __shared__ float4 runs[2][kWarps][32];
    __shared__ float2 ends[2][kWarps][32];
    const ScanArgs& a = ba.f;
    const int D = a.s.D, L = a.s.L, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t blocks = a.s.blocks(), spans = a.s.spans();
    const int64_t b = blockIdx.x / blocks, blk = blockIdx.x - b * blocks;
    const int c0 = (int)blk * kScanCh + 2 * lane, n = max(0, min(2, D - c0));
    float2 rate = load2<float>(a.rate, c0, n, false);
    rate = make_float2(-rate.x, -rate.y);
    float2 carry = ba.dh_final ? load2<float>(ba.dh_final, b * D + c0, n, false) : dup(0.0f), sum = dup(0.0f);
    int flip = 0;
    for (int64_t tile = spans - 1; tile >= 0; --tile, flip ^= 1) {
        const int t0 = (int)(tile * kScanSpan) + warp * kTok;
        float2 x[kTok], c[kTok], wr[kTok], wi[kTok], s[kTok], rs[kTok], lam[kTok], hp[kTok];
        unsigned first = 0, far = 0;  // bits of tokens; of channels of tokens
        float2 hh = dup(0.0f), pp = dup(1.0f);
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            const int t = t0 + j;
            const bool in = t < L;
            const int64_t at = (b * L + t) * D + c0;
            float2 r, g = dup(0.0f);
            if (PACK) {
                const int64_t row = (b * blocks + blk) * spans * kScanSpan + t;
                float2 v[3];
#pragma unroll
                for (int k = 0; k < (GATE ? 3 : 2); ++k) {
                    float w[2];
                    pack8::decode<2>(*reinterpret_cast<const pack8::Codes<2>*>(a.codes + k * a.code_step + row * kScanCh + 2 * lane),
                                     a.scales[k * a.scale_step + row * 2 + (lane >> 4)], w);
                    v[k] = make_float2(w[0], w[1]);
                }
                x[j] = v[0]; r = v[1];
                if (GATE) g = v[2];
            } else {
                x[j] = load2<IO>(a.x, at, in ? n : 0, pair);
                r = load2<IO>(a.r, at, in ? n : 0, pair);
                if (GATE) g = load2<IO>(a.g, at, in ? n : 0, pair);
            }
            wi[j] = GATE ? smaller_part2<IO>(g) : dup(0.0f);
            wr[j] = smaller_part2<IO>(r);
            const Decay d = decay<IO, UNIT, false>(open2(wr[j]), rate);
            c[j] = d.c;
            far |= d.far << 2 * j;
            rs[j] = UNIT ? inv_sqrt2<IO>(d.one) : dup(1.0f);
            s[j] = UNIT ? mul2(d.one, rs[j]) : dup(1.0f);
            lam[j] = load2<IO>(ba.d_h, at, in ? n : 0, pair);
            if (in && a.starts && a.starts[b * L + t]) {
                first |= 1u << j;
                s[j] = dup(1.0f);
                hh = mul2(open2(wi[j]), x[j]);
                pp = dup(0.0f);
            } else if (in) {
                hh = add2(fade<false>(hh, c[j], d.far), mul2(s[j], mul2(open2(wi[j]), x[j])));
                pp = fade<false>(pp, c[j], d.far);
            }
        }
        float2 v = dup(0.0f);
#pragma unroll
        for (int j = kTok - 1; j >= 0; --j) {
            if (t0 + j >= L) continue;
            v = add2(v, lam[j]);
            v = first >> j & 1 ? dup(0.0f) : fade<false>(v, c[j], far >> 2 * j);
        }
        runs[flip][warp][lane] = make_float4(pp.x, pp.y, hh.x, hh.y);
        ends[flip][warp][lane] = v;
        __syncthreads();
        float2 state = load2<float>(a.states, (b * spans + tile) * D + c0, n, false), in = carry;
        for (int w = 0; w < warp; ++w) {
            const float4 q = runs[flip][w][lane];
            state.x = q.x == 0.0f ? q.z : fmaf(q.x, state.x, q.z);
            state.y = q.y == 0.0f ? q.w : fmaf(q.y, state.y, q.w);
        }
        for (int w = kWarps - 1; w >= 0; --w) {
            const float4 q = runs[flip][w][lane];
            const float2 e = ends[flip][w][lane];
            if (w == warp) in = carry;
            carry.x = q.x == 0.0f ? e.x : fmaf(q.x, carry.x, e.x);
            carry.y = q.y == 0.0f ? e.y : fmaf(q.y, carry.y, e.y);
        }
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            hp[j] = state;
            if (t0 + j < L) state = first >> j & 1 ? mul2(open2(wi[j]), x[j]) : add2(fade<false>(state, c[j], far >> 2 * j), mul2(s[j], mul2(open2(wi[j]), x[j])));
        }
#pragma unroll
        for (int j = kTok - 1; j >= 0; --j) {
            if (t0 + j >= L) continue;
            const int64_t at = (b * L + t0 + j) * D + c0;
            in = add2(in, lam[j]);
            const float2 ls = mul2(in, s[j]), u = mul2(open2(wi[j]), x[j]);
            store2<IO>(ba.d_x, at, n, pair, mul2(ls, open2(wi[j])));
            if (GATE) store2<IO>(ba.d_g, at, n, pair, mul2(mul2(ls, u), closed2(wi[j])));
            const float2 al = fade<false>(in, c[j], far >> 2 * j);  // a lam
            float2 dl = dup(0.0f);
            if (!(first >> j & 1)) {
                float2 to = hp[j];
                if (UNIT) {
                    const float2 ur = mul2(u, rs[j]), au = fade<false>(ur, c[j], far >> 2 * j);
                    to = make_float2(to.x - au.x, to.y - au.y);
                }
                dl = mul2(al, to);
                sum = fma2(make_float2(-dl.x, -dl.y), open2(wr[j]), sum);
            }
            store2<IO>(ba.d_r, at, n, pair, mul2(mul2(dl, mul2(rate, open2(wr[j]))), closed2(wr[j])));
            in = first >> j & 1 ? dup(0.0f) : al;
        }
    }
    if (warp == 0) store2<float>(ba.dh_init, b * D + c0, n, false, carry);
    __syncthreads();
    ends[0][warp][lane] = sum;
    __syncthreads();
    if (warp != 0) return;
    sum = ends[0][0][lane];
    for (int w = 1; w < kWarps; ++w) sum = add2(sum, ends[0][w][lane]);
    store2<float>(ba.part, b * D + c0, n, false, sum);
}

__global__ void scan_rate_kernel(const float* part, float* d_rate, const int64_t rows, const int D) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= D) return;
    float y = 0.0f;
    for (int64_t i = 0; i < rows; ++i) y += part[i * D + c];
    d_rate[c] = y;
}

template <typename IO, bool GATE, bool UNIT> int launch(const ScanBwdArgs& b, bool pair, cudaStream_t st) {
    const ScanShape& s = b.f.s;
    const unsigned grid = (unsigned)(s.B * s.blocks());
    if (b.f.codes) scan_bwd_kernel<IO, GATE, UNIT, true><<<grid, kThreads, 0, st>>>(b, pair);
    else scan_bwd_kernel<IO, GATE, UNIT, false><<<grid, kThreads, 0, st>>>(b, pair);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return (int)e;
    scan_rate_kernel<<<(s.D + 63) / 64, 64, 0, st>>>(b.part, b.d_rate, (int64_t)s.B * scan_parts(s), s.D);
    return (int)cudaGetLastError();
}
template <typename IO> int dispatch(const ScanBwdArgs& b, bool pair, cudaStream_t st) {
    if (b.f.s.gate) return b.f.s.unit ? launch<IO, true, true>(b, pair, st) : launch<IO, true, false>(b, pair, st);
    return b.f.s.unit ? launch<IO, false, true>(b, pair, st) : launch<IO, false, false>(b, pair, st);
}

}  // namespace

int scan_bwd_launch(const ScanBwdArgs& b, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    uintptr_t all = 0;
    for (const void* p : {b.f.x, b.f.r, b.f.g, b.d_h, (const void*)b.d_x, (const void*)b.d_r, (const void*)b.d_g}) all |= reinterpret_cast<uintptr_t>(p);
    const bool pair = b.f.s.D % 2 == 0 && all % (b.f.s.f32 ? 8 : 4) == 0;
    return b.f.s.f32 ? dispatch<float>(b, pair, st) : dispatch<__nv_bfloat16>(b, pair, st);
}

}  // namespace e2ttt
