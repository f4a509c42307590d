// Gated delta rule, the walk over the chunks.  A warp owns 16 value rows of one sequence's state: the slice [16, dk] stays in its registers
// (64 of them at dk = 128) from the first token to the last, and the warps of a sequence never meet but for the tiles that they share.
// Per chunk of 32 tokens, rows = value rows:  P = V - b S K^T,  e = P T^T,  O = b S Q^T + u A^T,  S = b_end S + (D_end u) K.
// Each product's result is the next one's A operand in place.  The chunk's tiles (queries, keys, T, A, scalars; written by
// delta_prep.cu) arrive by bulk copies, several chunks ahead.
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

constexpr int kStages = 3;

template <int DK, int KT> constexpr int stage_bytes() { return 2 * KT * 64 * DK + kDeltaRecBytes; }

template <typename IO, int DK, int KT>
__global__ void __launch_bounds__(128) delta_fwd_kernel(const DeltaArgs a, const int warps) {
    extern __shared__ __align__(1024) char smem[];
    __shared__ uint64_t full[kStages];
    __shared__ int dead_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const DeltaShape& s = a.s;
    const int groups = (a.l.slices + warps - 1) / warps;  // CTAs per sequence
    const int64_t n = blockIdx.x / groups, nk = (n / s.H) * s.Hk + (n % s.H) / (s.H / s.Hk);
    const int slice = (int)(blockIdx.x % groups) * warps + warp;
    const bool active = slice < a.l.slices;
    const int nch = a.l.nch;
    sm100::WaitCtx wait{&dead_flag, reinterpret_cast<int*>(a.ws)};
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) sm100::mbar_init(&full[i], 1);
        dead_flag = 0;
        sm100::fence_mbar_init();
    }
    __syncthreads();
    const char* qk_src = a.ws + a.l.qk + (size_t)nk * nch * a.l.qk_bytes;
    const char* rec_src = a.ws + a.l.rec + (size_t)n * nch * a.l.rec_bytes;
    auto fetch = [&](int c) {  // one thread
        const uint32_t dst = sm100::smem_u32(smem) + (c % kStages) * stage_bytes<DK, KT>();
        uint64_t* bar = &full[c % kStages];
        sm100::mbar_expect_tx(bar, stage_bytes<DK, KT>());
        bulk_copy(dst, qk_src + (size_t)c * a.l.qk_bytes, 2 * KT * 64 * DK, bar);
        bulk_copy(dst + 2 * KT * 64 * DK, rec_src + (size_t)c * a.l.rec_bytes, kDeltaRecBytes, bar);
    };
    if (threadIdx.x == 0)
        for (int c = 0; c < kStages && c < nch; ++c) fetch(c);

    const int r0 = slice * 16 + g, r1 = r0 + 8;  // the lane's two value rows
    const bool ok0 = active && r0 < s.dv, ok1 = active && r1 < s.dv;
    float S[DK / 8][4];
#pragma unroll
    for (int j = 0; j < DK / 8; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int col = j * 8 + 2 * c4 + (x & 1);
            const bool ok = a.S_init && col < s.dk && (x < 2 ? ok0 : ok1);
            S[j][x] = ok ? a.S_init[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] : 0.0f;
        }
    const IO* v = reinterpret_cast<const IO*>(a.v) + (size_t)n * s.L * s.dv;
    IO* o = a.o ? reinterpret_cast<IO*>(a.o) + (size_t)n * s.L * s.dv : nullptr;
    auto load_v = [&](int c, float (&x)[4][4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (i & 1);
                x[j][i] = (t < s.L && (i < 2 ? ok0 : ok1)) ? to_f32(v[(size_t)t * s.dv + (i < 2 ? r0 : r1)]) : 0.0f;
            }
    };
    auto save_state = [&](int slot) {
        float* dst = reinterpret_cast<float*>(a.ws + a.l.S) + ((size_t)n * (a.l.nblk + 1) + slot) * a.l.dvp * DK;
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < DK / 8; ++j) {
            *reinterpret_cast<float2*>(dst + (size_t)r0 * DK + j * 8 + 2 * c4) = make_float2(S[j][0], S[j][1]);
            *reinterpret_cast<float2*>(dst + (size_t)r1 * DK + j * 8 + 2 * c4) = make_float2(S[j][2], S[j][3]);
            m = fmaxf(m, fmaxf(fmaxf(fabsf(S[j][0]), fabsf(S[j][1])), fmaxf(fabsf(S[j][2]), fabsf(S[j][3]))));
        }
        m = warp_max(m);
        if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.max_s)[((size_t)n * (a.l.nblk + 1) + slot) * a.l.slices + slice] = m;
    };
    auto save_tok = [&](size_t off, int c, const float (&x)[4][4]) {
        float* dst = reinterpret_cast<float*>(a.ws + off) + ((size_t)n * nch + c) * a.l.dvp * kDeltaChunk;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            *reinterpret_cast<float2*>(dst + r0 * kDeltaChunk + j * 8 + 2 * c4) = make_float2(x[j][0], x[j][1]);
            *reinterpret_cast<float2*>(dst + r1 * kDeltaChunk + j * 8 + 2 * c4) = make_float2(x[j][2], x[j][3]);
        }
    };
    float vn[4][4];
    load_v(0, vn);
    for (int c = 0; c < nch; ++c) {
        const int st = c % kStages;
        sm100::mbar_wait(&full[st], (c / kStages) & 1, wait, 901);
        if (active) {
            const uint32_t ks = sm100::smem_u32(smem) + st * stage_bytes<DK, KT>(), qs = ks + KT * 64 * DK, ts = qs + KT * 64 * DK, as = ts + 4096;
            const float* sc = reinterpret_cast<const float*>(smem + st * stage_bytes<DK, KT>() + 2 * KT * 64 * DK + 8192);
            if (a.save && (c & 1) == 0) save_state(c >> 1);
            // S K^T and S Q^T
            float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < DK / 8; ++j) {
                m0 = fmaxf(m0, fmaxf(fabsf(S[j][0]), fabsf(S[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(S[j][2]), fabsf(S[j][3])));
            }
            float s0, s1, i0, i1;
            pow2_scale(quad_max(m0), s0, i0);
            pow2_scale(quad_max(m1), s1, i1);
            float sk[4][4], sq[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) sk[j][x] = sq[j][x] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < DK / 16; ++kk) {
                uint32_t hi[4], lo[4];
                to_a(S[2 * kk], S[2 * kk + 1], s0, s1, hi, lo);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t b[4];
                    ldsm4(b, addr_nk<DK>(ks, 2 * h, kk, lane));
                    mma(sk[2 * h], hi, b[0], b[1]); mma(sk[2 * h + 1], hi, b[2], b[3]);
                    mma(sk[2 * h], lo, b[0], b[1]); mma(sk[2 * h + 1], lo, b[2], b[3]);
                    if (KT == 2) {
                        ldsm4(b, addr_nk<DK>(ks + 64 * DK, 2 * h, kk, lane));
                        mma(sk[2 * h], hi, b[0], b[1]); mma(sk[2 * h + 1], hi, b[2], b[3]);
                    }
                    ldsm4(b, addr_nk<DK>(qs, 2 * h, kk, lane));
                    mma(sq[2 * h], hi, b[0], b[1]); mma(sq[2 * h + 1], hi, b[2], b[3]);
                    mma(sq[2 * h], lo, b[0], b[1]); mma(sq[2 * h + 1], lo, b[2], b[3]);
                    if (KT == 2) {
                        ldsm4(b, addr_nk<DK>(qs + 64 * DK, 2 * h, kk, lane));
                        mma(sq[2 * h], hi, b[0], b[1]); mma(sq[2 * h + 1], hi, b[2], b[3]);
                    }
                }
            }
            // P = V - b S K^T; the values of the next chunk are on their way meanwhile
            float p[4][4];
            m0 = m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 bk = *reinterpret_cast<const float2*>(sc + kRecBk * 32 + j * 8 + 2 * c4);
                p[j][0] = fmaf(-sk[j][0] * i0, bk.x, vn[j][0]); p[j][1] = fmaf(-sk[j][1] * i0, bk.y, vn[j][1]);
                p[j][2] = fmaf(-sk[j][2] * i1, bk.x, vn[j][2]); p[j][3] = fmaf(-sk[j][3] * i1, bk.y, vn[j][3]);
                m0 = fmaxf(m0, fmaxf(fabsf(p[j][0]), fabsf(p[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(p[j][2]), fabsf(p[j][3])));
            }
            if (c + 1 < nch) load_v(c + 1, vn);
            const float tinv = sc[kRecHead * 32 + 1], ainv = sc[kRecHead * 32 + 2], bend = sc[kRecHead * 32 + 0];
            float e[4][4], in[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) e[j][x] = in[j][x] = 0.0f;
            // x M^T for a lower M [t][i] (two terms)
            auto lower = [&](float (&acc)[4][4], uint32_t tile, const float (&x)[4][4], float f0, float f1) {
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    uint32_t hi[4], lo[4];
                    to_a(x[2 * kk], x[2 * kk + 1], f0, f1, hi, lo);
#pragma unroll
                    for (int h = kk; h < 2; ++h) {
                        uint32_t bh[4], bl[4];
                        ldsm4(bh, addr_nk<32>(tile, 2 * h, kk, lane));
                        ldsm4(bl, addr_nk<32>(tile + 2048, 2 * h, kk, lane));
                        mma(acc[2 * h], hi, bh[0], bh[1]); mma(acc[2 * h + 1], hi, bh[2], bh[3]);
                        mma(acc[2 * h], lo, bh[0], bh[1]); mma(acc[2 * h + 1], lo, bh[2], bh[3]);
                        mma(acc[2 * h], hi, bl[0], bl[1]); mma(acc[2 * h + 1], hi, bl[2], bl[3]);
                    }
                }
            };
            float p0, p1, q0, q1;
            pow2_scale(quad_max(m0), p0, q0);
            pow2_scale(quad_max(m1), p1, q1);
            lower(e, ts, p, p0, p1);
            q0 *= tinv; q1 *= tinv;
            // u = eta e
            float u[4][4];
            m0 = m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 et = *reinterpret_cast<const float2*>(sc + kRecEta * 32 + j * 8 + 2 * c4);
                e[j][0] *= q0; e[j][1] *= q0; e[j][2] *= q1; e[j][3] *= q1;
                u[j][0] = e[j][0] * et.x; u[j][1] = e[j][1] * et.y; u[j][2] = e[j][2] * et.x; u[j][3] = e[j][3] * et.y;
                m0 = fmaxf(m0, fmaxf(fabsf(u[j][0]), fabsf(u[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(u[j][2]), fabsf(u[j][3])));
            }
            if (a.save) {
                const float m = warp_max(fmaxf(m0, m1));
                if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.max_u)[((size_t)n * nch + c) * a.l.slices + slice] = m;
                save_tok(a.l.e, c, e);
            }
            pow2_scale(quad_max(m0), p0, q0);
            pow2_scale(quad_max(m1), p1, q1);
            // S = b_end S + (D_end u) K: the sum of the chunk apart from the state (the MMAs truncate what they add to), then one rounding
            float w0 = 0.0f, w1 = 0.0f, w[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 de = *reinterpret_cast<const float2*>(sc + kRecDend * 32 + j * 8 + 2 * c4);
                w[j][0] = u[j][0] * de.x; w[j][1] = u[j][1] * de.y; w[j][2] = u[j][2] * de.x; w[j][3] = u[j][3] * de.y;
                w0 = fmaxf(w0, fmaxf(fabsf(w[j][0]), fabsf(w[j][1])));
                w1 = fmaxf(w1, fmaxf(fabsf(w[j][2]), fabsf(w[j][3])));
            }
            float f0, f1, h0, h1;
            pow2_scale(quad_max(w0), f0, h0);
            pow2_scale(quad_max(w1), f1, h1);
            uint32_t wh[2][4], wl[2][4];
            to_a(w[0], w[1], f0, f1, wh[0], wl[0]);
            to_a(w[2], w[3], f0, f1, wh[1], wl[1]);
#pragma unroll
            for (int j2 = 0; j2 < DK / 16; ++j2) {
                float x[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    uint32_t b[4];
                    ldsm4_t(b, addr_kn<DK>(ks, 2 * j2, kk, lane));
                    mma(x[0], wh[kk], b[0], b[1]); mma(x[1], wh[kk], b[2], b[3]);
                    mma(x[0], wl[kk], b[0], b[1]); mma(x[1], wl[kk], b[2], b[3]);
                    if (KT == 2) {
                        ldsm4_t(b, addr_kn<DK>(ks + 64 * DK, 2 * j2, kk, lane));
                        mma(x[0], wh[kk], b[0], b[1]); mma(x[1], wh[kk], b[2], b[3]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float (&d)[4] = S[2 * j2 + i];
                    d[0] = fmaf(x[i][0], h0, bend * d[0]); d[1] = fmaf(x[i][1], h0, bend * d[1]);
                    d[2] = fmaf(x[i][2], h1, bend * d[2]); d[3] = fmaf(x[i][3], h1, bend * d[3]);
                }
            }
            // O = b S Q^T + u A^T (off the chain of the state)
            lower(in, as, u, p0, p1);
            q0 *= ainv; q1 *= ainv;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 bq = *reinterpret_cast<const float2*>(sc + kRecBq * 32 + j * 8 + 2 * c4);
                in[j][0] = fmaf(sq[j][0] * i0, bq.x, in[j][0] * q0); in[j][1] = fmaf(sq[j][1] * i0, bq.y, in[j][1] * q0);
                in[j][2] = fmaf(sq[j][2] * i1, bq.x, in[j][2] * q1); in[j][3] = fmaf(sq[j][3] * i1, bq.y, in[j][3] * q1);
            }
            if (a.save) save_tok(a.l.o, c, in);
            if (o) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (x & 1);
                        if (t < s.L && (x < 2 ? ok0 : ok1)) o[(size_t)t * s.dv + (x < 2 ? r0 : r1)] = from_f32<IO>(in[j][x]);
                    }
            }
        }
        __syncthreads();  // every warp has read the stage
        if (threadIdx.x == 0 && c + kStages < nch) fetch(c + kStages);
    }
    if (!active) return;
    if (a.save) save_state(a.l.nblk);
    if (a.S_final) {
#pragma unroll
        for (int j = 0; j < DK / 8; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int col = j * 8 + 2 * c4 + (x & 1);
                if (col < s.dk && (x < 2 ? ok0 : ok1)) a.S_final[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] = S[j][x];
            }
    }
}

template <typename IO, int DK, int KT> int launch(const DeltaArgs& a, cudaStream_t st) {
    constexpr int bytes = kStages * stage_bytes<DK, KT>();
    auto kernel = delta_fwd_kernel<IO, DK, KT>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return (int)e;
    // slices per CTA: they share the tiles in shared memory, but a warp with a scheduler of its own walks fastest
    int w = 4;
    while (w > 1 && a.l.N * ((a.l.slices + w - 1) / w) < 96) w >>= 1;
    const unsigned grid = (unsigned)(a.l.N * ((a.l.slices + w - 1) / w));
    kernel<<<grid, w * 32, bytes, st>>>(a, w);
    return (int)cudaGetLastError();
}

}  // namespace

int delta_fwd_launch(const DeltaArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.s.f32) return a.l.DK == 64 ? launch<float, 64, 2>(a, st) : launch<float, 128, 2>(a, st);
    return a.l.DK == 64 ? launch<__nv_bfloat16, 64, 1>(a, st) : launch<__nv_bfloat16, 128, 1>(a, st);
}

}  // namespace e2ttt
