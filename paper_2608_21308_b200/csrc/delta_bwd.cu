// Gated delta rule, reverse pass.  With X the adjoint of the state behind a chunk and Z = (I + eta strict(D K K^T))^-T dU:
//   dU = A^T dO + D_end X K,   dP = eta Z = dV,   X_before = b_end X + scale (b dO) Q^T - (b dP) K^T            (delta_chain_kernel)
//   dQ = (D dO^T U) K + scale b S_0^T dO,   dK = (D dO^T U)^T Q - (W + W^T) K - b S_0^T dP + D_end X^T U,  W = strict(D dP^T U)   (delta_qk_kernel)
//   d eta = Z . e,   d log_gamma_t = sum over s >= t (o_s . do_s - v_s . dv_s) + <X, S> at the end of the sum         (delta_gate_kernel)
// The last line is the scaling of everything before token t by g_t: outputs and state are linear in the start state and the values, so
// no difference of nearly equal sums over keys is formed.  Sums run over 128 tokens, <X, S> is taken behind each of them.
// The chain walks the chunks from the last to the first as the forward does, a warp per 16 value rows; dQ and dK contract over the
// value rows of all warps and are left to a kernel that takes the blocks side by side.
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

constexpr int kStages = 3;

template <int DK, int KT> constexpr int stage_bytes() { return 2 * KT * 64 * DK + kDeltaRecBytes; }

// sum of 8 values over the eight lanes that differ in bits 2..4: lane gets the sum of v[lane >> 2]
__device__ __forceinline__ float sum_rows(const float (&v)[8], int lane) {
    float a[4], b[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float keep = (lane & 16) ? v[j + 4] : v[j], give = (lane & 16) ? v[j] : v[j + 4];
        a[j] = keep + __shfl_xor_sync(kAll, give, 16);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float keep = (lane & 8) ? a[j + 2] : a[j], give = (lane & 8) ? a[j] : a[j + 2];
        b[j] = keep + __shfl_xor_sync(kAll, give, 8);
    }
    const float keep = (lane & 4) ? b[1] : b[0], give = (lane & 4) ? b[0] : b[1];
    return keep + __shfl_xor_sync(kAll, give, 4);
}

template <typename IO, int DK, int KT>
__global__ void __launch_bounds__(128) delta_chain_kernel(const DeltaBwdArgs ba, const int warps) {
    extern __shared__ __align__(1024) char smem[];
    __shared__ uint64_t full[kStages];
    __shared__ int dead_flag;
    const DeltaArgs& a = ba.f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const DeltaShape& s = a.s;
    const int groups = (a.l.slices + warps - 1) / warps;
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
    const char* rec_src = a.ws + a.l.rec + (size_t)n * nch * a.l.rec_bytes + kDeltaRecSkip;
    auto fetch = [&](int i) {  // the i-th chunk from the end
        const int c = nch - 1 - i;
        const uint32_t dst = sm100::smem_u32(smem) + (i % kStages) * stage_bytes<DK, KT>();
        uint64_t* bar = &full[i % kStages];
        sm100::mbar_expect_tx(bar, stage_bytes<DK, KT>());
        bulk_copy(dst, qk_src + (size_t)c * a.l.qk_bytes, 2 * KT * 64 * DK, bar);
        bulk_copy(dst + 2 * KT * 64 * DK, rec_src + (size_t)c * a.l.rec_bytes, kDeltaRecBytes, bar);
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < kStages && i < nch; ++i) fetch(i);

    const int r0 = slice * 16 + g, r1 = r0 + 8;
    const bool ok0 = active && r0 < s.dv, ok1 = active && r1 < s.dv;
    float X[DK / 8][4];
#pragma unroll
    for (int j = 0; j < DK / 8; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int col = j * 8 + 2 * c4 + (x & 1);
            const bool ok = ba.dS_final && col < s.dk && (x < 2 ? ok0 : ok1);
            X[j][x] = ok ? ba.dS_final[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] : 0.0f;
        }
    const size_t seq = (size_t)n * s.L * s.dv;
    const IO* v = reinterpret_cast<const IO*>(a.v) + seq;
    const IO* d_o = reinterpret_cast<const IO*>(ba.d_o) + seq;
    IO* dv = reinterpret_cast<IO*>(ba.dv) + seq;
    auto load_tok = [&](const IO* p, int c, float (&x)[4][4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (i & 1);
                x[j][i] = (t < s.L && (i < 2 ? ok0 : ok1)) ? to_f32(p[(size_t)t * s.dv + (i < 2 ? r0 : r1)]) : 0.0f;
            }
    };
    float don[4][4];
    load_tok(d_o, nch - 1, don);
    for (int i = 0; i < nch; ++i) {
        const int c = nch - 1 - i, st = i % kStages;
        sm100::mbar_wait(&full[st], (i / kStages) & 1, wait, 902);
        if (active) {
            const uint32_t ks = sm100::smem_u32(smem) + st * stage_bytes<DK, KT>(), qs = ks + KT * 64 * DK, as = qs + KT * 64 * DK + 1024, ts = as + 4096;
            const float* sc = reinterpret_cast<const float*>(smem + st * stage_bytes<DK, KT>() + 2 * KT * 64 * DK);
            const int blk = c >> 1;
            const bool block_end = (c & 1) || c == nch - 1;
            if (block_end && ((blk + 1) % kDeltaSuper == 0 || blk + 1 == a.l.nblk)) {  // <X, S> behind a superblock
                const int lo = delta_lo_slot(blk + 1, a.l.nblk, s.f32);
                const size_t at = ((size_t)n * (a.l.nblk + 1) + blk + 1) * a.l.slices + slice;
                const size_t at_lo = s.f32 ? at : ((size_t)n * a.l.nsup + lo) * a.l.slices + slice;
                const uint4* hi4 = reinterpret_cast<const uint4*>(a.ws + a.l.S + at * a.l.state_bytes);
                const uint4* lo4 = reinterpret_cast<const uint4*>(a.ws + a.l.S_lo + at_lo * a.l.state_bytes);
                float h = 0.0f;
#pragma unroll
                for (int kk = 0; kk < DK / 16; ++kk) {
                    const uint4 u = hi4[kk * 32 + lane], v2 = lo4[kk * 32 + lane];
                    const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v2.x, v2.y, v2.z, v2.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float s0, s1;
                        join_terms(uw[r], vw[r], s0, s1);
                        const float (&x)[4] = X[2 * kk + (r >> 1)];
                        h = fmaf(x[2 * (r & 1)], s0, h);
                        h = fmaf(x[2 * (r & 1) + 1], s1, h);
                    }
                }
                h = warp_sum(h) * reinterpret_cast<const float*>(a.ws + a.l.s_inv)[at];
                if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.hx)[((size_t)n * a.l.nsup + blk / kDeltaSuper) * a.l.slices + slice] = h;
            }
            float xk[4][4], in[4][4], z[4][4], d_out[4][4];
            float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) { xk[j][x] = in[j][x] = z[j][x] = 0.0f; d_out[j][x] = don[j][x]; }
            if (c > 0) load_tok(d_o, c - 1, don);
            // X K^T
#pragma unroll
            for (int j = 0; j < DK / 8; ++j) {
                m0 = fmaxf(m0, fmaxf(fabsf(X[j][0]), fabsf(X[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(X[j][2]), fabsf(X[j][3])));
            }
            float s0, i0;
            pow2_scale(warp_max(fmaxf(m0, m1)), s0, i0);
            const size_t at_x = ((size_t)n * (a.l.nblk + 1) + blk) * a.l.slices + slice;
            uint4* x_out = reinterpret_cast<uint4*>(a.ws + a.l.X + at_x * a.l.state_bytes * KT);
            if (block_end && lane == 0) reinterpret_cast<float*>(a.ws + a.l.x_inv)[at_x] = i0;
#pragma unroll
            for (int kk = 0; kk < DK / 16; ++kk) {
                uint32_t hi[4], lo[4];
                to_a(X[2 * kk], X[2 * kk + 1], s0, s0, hi, lo);
                if (block_end) {
                    x_out[kk * 32 + lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    if (KT == 2) x_out[(DK / 16 + kk) * 32 + lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t b[4];
                    ldsm4(b, addr_nk<DK>(ks, 2 * h, kk, lane));
                    mma(xk[2 * h], hi, b[0], b[1]); mma(xk[2 * h + 1], hi, b[2], b[3]);
                    mma(xk[2 * h], lo, b[0], b[1]); mma(xk[2 * h + 1], lo, b[2], b[3]);
                    if (KT == 2) {
                        ldsm4(b, addr_nk<DK>(ks + 64 * DK, 2 * h, kk, lane));
                        mma(xk[2 * h], hi, b[0], b[1]); mma(xk[2 * h + 1], hi, b[2], b[3]);
                    }
                }
            }
            // y M for a lower M [t][i] (two terms): contraction over t >= i
            auto lower_t = [&](float (&acc)[4][4], uint32_t tile, const float (&y)[4][4], float f0, float f1) {
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    uint32_t hi[4], lo[4];
                    to_a(y[2 * kk], y[2 * kk + 1], f0, f1, hi, lo);
#pragma unroll
                    for (int h = 0; h <= kk; ++h) {
                        uint32_t bh[4], bl[4];
                        ldsm4_t(bh, addr_kn<32>(tile, 2 * h, kk, lane));
                        ldsm4_t(bl, addr_kn<32>(tile + 2048, 2 * h, kk, lane));
                        mma(acc[2 * h], hi, bh[0], bh[1]); mma(acc[2 * h + 1], hi, bh[2], bh[3]);
                        mma(acc[2 * h], lo, bh[0], bh[1]); mma(acc[2 * h + 1], lo, bh[2], bh[3]);
                        mma(acc[2 * h], hi, bl[0], bl[1]); mma(acc[2 * h + 1], hi, bl[2], bl[3]);
                    }
                }
            };
            m0 = m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m0 = fmaxf(m0, fmaxf(fabsf(d_out[j][0]), fabsf(d_out[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(d_out[j][2]), fabsf(d_out[j][3])));
            }
            m0 = quad_max(m0); m1 = quad_max(m1);
            const size_t at_max = ((size_t)n * nch + c) * a.l.slices + slice;
            {
                const float m = warp_max(fmaxf(m0, m1));
                if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.max_do)[at_max] = m;
            }
            float f0, f1, h0, h1;
            pow2_scale(m0, f0, h0);
            pow2_scale(m1, f1, h1);
            lower_t(in, as, d_out, f0, f1);
            const float ainv = sc[kRecHead * 32 + kHeadAr], rinv = sc[kRecHead * 32 + kHeadR], bend = sc[kRecHead * 32 + kHeadEnd];
            // dU, then Z
            h0 *= ainv; h1 *= ainv;
            m0 = m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 de = *reinterpret_cast<const float2*>(sc + kRecDend * 32 + j * 8 + 2 * c4);
                in[j][0] = fmaf(xk[j][0] * i0, de.x, in[j][0] * h0); in[j][1] = fmaf(xk[j][1] * i0, de.y, in[j][1] * h0);
                in[j][2] = fmaf(xk[j][2] * i0, de.x, in[j][2] * h1); in[j][3] = fmaf(xk[j][3] * i0, de.y, in[j][3] * h1);
                m0 = fmaxf(m0, fmaxf(fabsf(in[j][0]), fabsf(in[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(in[j][2]), fabsf(in[j][3])));
            }
            pow2_scale(quad_max(m0), f0, h0);
            pow2_scale(quad_max(m1), f1, h1);
            lower_t(z, ts, in, f0, f1);
            h0 *= rinv; h1 *= rinv;
#pragma unroll
            for (int j = 0; j < 4; ++j) { z[j][0] *= h0; z[j][1] *= h0; z[j][2] *= h1; z[j][3] *= h1; }
            // sums over the slice's value rows for d eta and d log_gamma
            {
                float part[8], vv[4][4];
                const uint4* ef = reinterpret_cast<const uint4*>(a.ws + a.l.e) + at_max * 128;
                const float e_inv = reinterpret_cast<const float*>(a.ws + a.l.e_inv)[at_max];
                const float4* ov = reinterpret_cast<const float4*>(a.ws + a.l.o) + at_max * 128;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const uint4 u = ef[kk * 32 + lane], w = ef[(2 + kk) * 32 + lane];
                    const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, ww[4] = {w.x, w.y, w.z, w.w};
                    float e[4][2];
#pragma unroll
                    for (int r = 0; r < 4; ++r) join_terms(uw[r], ww[r], e[r][0], e[r][1]);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const float (&zz)[4] = z[2 * kk + j];
                            part[4 * kk + 2 * j + y] = fmaf(zz[y], e[2 * j][y], zz[2 + y] * e[2 * j + 1][y]) * e_inv;
                        }
                }
                // lane 4 g + c4 holds the sum of value g of its c4 group: token (g >> 1) * 8 + 2 c4 + (g & 1)
                const size_t at = at_max * kDeltaChunk + (g >> 1) * 8 + 2 * c4 + (g & 1);
                reinterpret_cast<float*>(a.ws + a.l.part_eta)[at] = sum_rows(part, lane);
                load_tok(v, c, vv);
                float w = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 et = *reinterpret_cast<const float2*>(sc + kRecEta * 32 + j * 8 + 2 * c4);
                    const float4 o4 = ov[j * 32 + lane];
                    z[j][0] *= et.x; z[j][1] *= et.y; z[j][2] *= et.x; z[j][3] *= et.y;  // dP = dV
                    part[2 * j] = o4.x * d_out[j][0] - vv[j][0] * z[j][0] + (o4.z * d_out[j][2] - vv[j][2] * z[j][2]);
                    part[2 * j + 1] = o4.y * d_out[j][1] - vv[j][1] * z[j][1] + (o4.w * d_out[j][3] - vv[j][3] * z[j][3]);
                    w = fmaxf(w, fmaxf(fmaxf(fabsf(z[j][0]), fabsf(z[j][1])), fmaxf(fabsf(z[j][2]), fabsf(z[j][3]))));
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (x & 1);
                        if (t < s.L && (x < 2 ? ok0 : ok1)) dv[(size_t)t * s.dv + (x < 2 ? r0 : r1)] = from_f32<IO>(z[j][x]);
                    }
                }
                reinterpret_cast<float*>(a.ws + a.l.part_gate)[at] = sum_rows(part, lane);
                float sp, ip;
                pow2_scale(warp_max(w), sp, ip);
                uint4* dst = reinterpret_cast<uint4*>(a.ws + a.l.dp) + at_max * 64 * KT;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    uint32_t hi[4], lo[4];
                    to_a(z[2 * kk], z[2 * kk + 1], sp, sp, hi, lo);
                    dst[kk * 32 + lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    if (KT == 2) dst[(2 + kk) * 32 + lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.dp_inv)[at_max] = ip;
            }
            // X = b_end X + (dO b scale) Q - (dP b) K
            m0 = m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 bq = *reinterpret_cast<const float2*>(sc + kRecBq * 32 + j * 8 + 2 * c4);
                const float2 bk = *reinterpret_cast<const float2*>(sc + kRecBk * 32 + j * 8 + 2 * c4);
                d_out[j][0] *= bq.x; d_out[j][1] *= bq.y; d_out[j][2] *= bq.x; d_out[j][3] *= bq.y;
                z[j][0] *= -bk.x; z[j][1] *= -bk.y; z[j][2] *= -bk.x; z[j][3] *= -bk.y;
                m0 = fmaxf(m0, fmaxf(fmaxf(fabsf(z[j][0]), fabsf(z[j][1])), fmaxf(fabsf(d_out[j][0]), fabsf(d_out[j][1]))));
                m1 = fmaxf(m1, fmaxf(fmaxf(fabsf(z[j][2]), fabsf(z[j][3])), fmaxf(fabsf(d_out[j][2]), fabsf(d_out[j][3]))));
            }
            pow2_scale(quad_max(m0), f0, h0);
            pow2_scale(quad_max(m1), f1, h1);
            uint32_t qh[2][4], ql[2][4], ph[2][4], pl[2][4];
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                to_a(d_out[2 * kk], d_out[2 * kk + 1], f0, f1, qh[kk], ql[kk]);
                to_a(z[2 * kk], z[2 * kk + 1], f0, f1, ph[kk], pl[kk]);
            }
#pragma unroll
            for (int j2 = 0; j2 < DK / 16; ++j2) {
                float x[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    uint32_t b[4];
                    ldsm4_t(b, addr_kn<DK>(ks, 2 * j2, kk, lane));
                    mma(x[0], ph[kk], b[0], b[1]); mma(x[1], ph[kk], b[2], b[3]);
                    mma(x[0], pl[kk], b[0], b[1]); mma(x[1], pl[kk], b[2], b[3]);
                    if (KT == 2) {
                        ldsm4_t(b, addr_kn<DK>(ks + 64 * DK, 2 * j2, kk, lane));
                        mma(x[0], ph[kk], b[0], b[1]); mma(x[1], ph[kk], b[2], b[3]);
                    }
                    ldsm4_t(b, addr_kn<DK>(qs, 2 * j2, kk, lane));
                    mma(x[0], qh[kk], b[0], b[1]); mma(x[1], qh[kk], b[2], b[3]);
                    mma(x[0], ql[kk], b[0], b[1]); mma(x[1], ql[kk], b[2], b[3]);
                    if (KT == 2) {
                        ldsm4_t(b, addr_kn<DK>(qs + 64 * DK, 2 * j2, kk, lane));
                        mma(x[0], qh[kk], b[0], b[1]); mma(x[1], qh[kk], b[2], b[3]);
                    }
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float (&d)[4] = X[2 * j2 + y];
                    d[0] = fmaf(x[y][0], h0, bend * d[0]); d[1] = fmaf(x[y][1], h0, bend * d[1]);
                    d[2] = fmaf(x[y][2], h1, bend * d[2]); d[3] = fmaf(x[y][3], h1, bend * d[3]);
                }
            }
        }
        __syncthreads();
        if (threadIdx.x == 0 && i + kStages < nch) fetch(i + kStages);
    }
    if (!active) return;
#pragma unroll
    for (int j = 0; j < DK / 8; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int col = j * 8 + 2 * c4 + (x & 1);
            if (col < s.dk && (x < 2 ? ok0 : ok1)) ba.dS_init[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] = X[j][x];
        }
}

// d eta and d log_gamma from the slices' sums: a CTA per superblock of 128 tokens, a warp per chunk, lane = token.  Sums of many terms in 64 bits:
// what is left of them counts
__global__ void __launch_bounds__(kDeltaSuper * 64) delta_gate_kernel(const DeltaBwdArgs ba) {
    __shared__ double total[2 * kDeltaSuper];
    const DeltaArgs& a = ba.f;
    const int64_t item = blockIdx.x, n = item / a.l.nsup;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = (int)(item % a.l.nsup) * kDeltaSuper * 2, c = first + warp;
    const int last = min(a.l.nch, first + kDeltaSuper * 2) - 1;
    float de = 0.0f, dg = 0.0f;
    if (c <= last) {
        const size_t at = ((size_t)n * a.l.nch + c) * a.l.slices * kDeltaChunk + lane;
#pragma unroll 4
        for (int i = 0; i < a.l.slices; ++i) {
            de += reinterpret_cast<const float*>(a.ws + a.l.part_eta)[at + i * kDeltaChunk];
            dg += reinterpret_cast<const float*>(a.ws + a.l.part_gate)[at + i * kDeltaChunk];
        }
    }
    double sum = dg;
#pragma unroll
    for (int i = 1; i < 32; i <<= 1) {  // suffix sums
        const double y = __shfl_down_sync(kAll, sum, i);
        if (lane + i < 32) sum += y;
    }
    if (lane == 0) total[warp] = sum;
    __syncthreads();
    if (c > last) return;
    const float* hx = reinterpret_cast<const float*>(a.ws + a.l.hx) + (size_t)item * a.l.slices;
    for (int i = 0; i < a.l.slices; ++i) sum += hx[i];
    for (int i = warp + 1; i <= last - first; ++i) sum += total[i];
    const int t = c * kDeltaChunk + lane;
    if (t < a.s.L) {
        const size_t out = (size_t)n * a.s.L + t;
        ba.d_eta[out] = de;
        ba.d_log_gamma[out] = a.log_gamma[out] < -104.0f ? 0.0f : (float)sum;  // a decay that is 0 in 32 bits has none
    }
}

// ---- dQ and dK ----------------------------------------------------------------------------------------------------
// A CTA takes 64 tokens of one query / key head and adds up the value heads of its group.  Sixteen warps: 16 tokens times a quarter of the key
// columns each.  The value rows come through shared memory ROWS at a time, with S_0 (dQ's and dK's first part, both token-by-token matrices) and
// again with X; what the chains left in fragment order goes into tiles of rows here, at one scale for all slices.  With bf16 I/O one term of every
// operand serves: dQ and dK are off by 2^-11 of their terms before they are rounded to 2^-8.
template <int DK, int KT> constexpr int qk_rows() { return KT == 1 ? 128 : 32; }
template <int DK, int KT> constexpr int qk_smem() {
    return 2 * KT * 128 * DK + KT * qk_rows<DK, KT>() * (2 * DK + 3 * 128) + 2 * KT * 8192 + 64 * 8 + 3 * 256 + 256;
}

template <typename IO, int DK, int KT>
__global__ void __launch_bounds__(512, 1) delta_qk_kernel(const DeltaBwdArgs ba, const bool vec) {
    extern __shared__ __align__(1024) char smem[];
    constexpr int ROWS = qk_rows<DK, KT>(), SL = ROWS / 16;  // value rows and slices at a time
    constexpr int TS = ROWS * DK * 2, TT = ROWS * 128;       // bytes of a term: state tile [ROWS][DK]; token tiles [ROWS][64], [64][ROWS]
    const DeltaArgs& a = ba.f;
    const DeltaShape& s = a.s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c4 = lane & 3;
    const int tw = warp >> 2, hw = warp & 3;
    const int64_t nk = blockIdx.x / a.l.nblk;
    const int blk = (int)(blockIdx.x % a.l.nblk), t0 = blk * kDeltaBlock, r = s.H / s.Hk;
    char* kq = smem;                    // K, then Q: [64][DK]
    char* st_s = kq + 2 * KT * 128 * DK;  // S or X
    char* st_o = st_s + KT * TS;        // dO [64][ROWS]
    char* st_u = st_o + KT * TT;        // e [ROWS][64]
    char* st_p = st_u + KT * TT;        // dP [ROWS][64]
    char* mat = st_p + KT * TT;         // sigma, then kappa + kappa^T
    double* run = reinterpret_cast<double*>(mat + 2 * KT * 8192);  // 64
    float* bt = reinterpret_cast<float*>(run + 64);                // 64
    float* dend = bt + 64;                                         // 64, times eta
    float* eta = dend + 64;                                        // 64
    float* red = eta + 64;                                         // 32, and the scales
    const uint32_t ks = sm100::smem_u32(kq), qs = ks + KT * 128 * DK, ss = sm100::smem_u32(st_s), os = sm100::smem_u32(st_o),
                   us = sm100::smem_u32(st_u), ps = sm100::smem_u32(st_p), ms = sm100::smem_u32(mat);
    const int nchunks = min(2, a.l.nch - 2 * blk);
    auto times_half = [](uint32_t x, __half2 y) {
        const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&x), y);
        return *reinterpret_cast<const uint32_t*>(&z);
    };
    // the two chunks' tiles at one scale
    float ik, iq;
    {
        const int64_t n0 = (nk / s.Hk) * s.H + (nk % s.Hk) * r;
        const float* h0 = reinterpret_cast<const float*>(a.ws + a.l.rec + ((size_t)n0 * a.l.nch + 2 * blk) * a.l.rec_bytes + 8192) + kRecHead * 32;
        const float* h1 = nchunks > 1 ? h0 + a.l.rec_bytes / 4 : h0;
        ik = fmaxf(h0[kHeadK], h1[kHeadK]); iq = fmaxf(h0[kHeadQ], h1[kHeadQ]);
        const float f[2][2] = {{h0[kHeadK] / ik, h0[kHeadQ] / iq}, {h1[kHeadK] / ik, h1[kHeadQ] / iq}};  // powers of two, at most 1
        constexpr int P = DK / 8;
        for (int i = tid; i < 2 * KT * 64 * P; i += 512) {
            const int piece = i % P, row = (i / P) % 64, term = (i / P / 64) % KT, which = i / P / 64 / KT;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (row / 32 < nchunks) {
                const char* src = a.ws + a.l.qk + ((size_t)nk * a.l.nch + 2 * blk + row / 32) * a.l.qk_bytes;
                x = *reinterpret_cast<const uint4*>(src + (which * KT + term) * 64 * DK + ((row & 31) * P + piece) * 16);
                const float y = f[row / 32][which];
                if (y != 1.0f) {
                    const __half2 m = __float2half2_rn(y);
                    x = make_uint4(times_half(x.x, m), times_half(x.y, m), times_half(x.z, m), times_half(x.w, m));
                }
            }
            *reinterpret_cast<uint4*>(kq + which * KT * 128 * DK + term * 128 * DK + (row * P + piece) * 16) = x;
        }
    }
    constexpr int NT = DK / 32;  // n-tiles of a warp's quarter of the columns
    float tq[NT][4], tk[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) tq[j][x] = tk[j][x] = 0.0f;
    const int row0 = tw * 16 + g, row1 = row0 + 8;
    for (int hd = 0; hd < r; ++hd) {
        const int64_t n = (nk / s.Hk) * s.H + (nk % s.Hk) * r + hd;
        __syncthreads();
        if (tid < 32) {  // decays and learning rates of the 64 tokens
            double sum[2];
            float et[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int t = t0 + 2 * lane + k;
                float lg = t < s.L ? a.log_gamma[(size_t)n * s.L + t] : 0.0f;
                if (lg < -1000.0f) lg = -1000.0f;
                sum[k] = (double)lg;
                et[k] = t < s.L ? a.eta[(size_t)n * s.L + t] : 0.0f;
            }
            sum[1] += sum[0];
            double acc = sum[1];
#pragma unroll
            for (int i = 1; i < 32; i <<= 1) {
                const double y = __shfl_up_sync(kAll, acc, i);
                if (lane >= i) acc += y;
            }
            const double end = __shfl_sync(kAll, acc, 31), before = acc - sum[1];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const double x = before + sum[k];
                run[2 * lane + k] = x;
                bt[2 * lane + k] = expf((float)x);
                dend[2 * lane + k] = expf((float)(end - x)) * et[k];
                eta[2 * lane + k] = et[k];
            }
        } else if (tid < 64) {  // the largest of the slices' scales; lane = slice and chunk
            const int sl = lane & 7, ch = lane >> 3;
            const bool ok = sl < a.l.slices;
            const size_t at = ((size_t)n * a.l.nch + 2 * blk + ch) * a.l.slices + sl;
            const bool tok = ok && ch < nchunks;
            const float iu = warp_most(tok ? reinterpret_cast<const float*>(a.ws + a.l.e_inv)[at] : 0.0f);
            const float ip = warp_most(tok ? reinterpret_cast<const float*>(a.ws + a.l.dp_inv)[at] : 0.0f);
            const float mo = warp_max(tok ? reinterpret_cast<const float*>(a.ws + a.l.max_do)[at] : 0.0f);
            const size_t at_s = ((size_t)n * (a.l.nblk + 1) + blk) * a.l.slices + sl;
            const float iS = warp_most(ok ? reinterpret_cast<const float*>(a.ws + a.l.s_inv)[at_s] : 0.0f);
            const float iX = warp_most(ok ? reinterpret_cast<const float*>(a.ws + a.l.x_inv)[at_s] : 0.0f);
            float so, io;
            pow2_scale(mo, so, io);
            if (lane == 0) { red[32] = iu; red[33] = ip; red[34] = so; red[35] = io; red[36] = iS; red[37] = iX; }
        }
        __syncthreads();
        const float iu = red[32], ip = red[33], so = red[34], io = red[35], iS = red[36], iX = red[37];
        // fragments [16 value rows][16 columns] of a slice to rows of a tile
        auto put = [&](char* tile, int cols, int row, int piece, const uint4& x, float ratio) {
            const __half2 m = __float2half2_rn(ratio);
            const uint32_t w[4] = {times_half(x.x, m), times_half(x.y, m), times_half(x.z, m), times_half(x.w, m)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = row + (i & 1) * 8, pp = piece + (i >> 1);
                const uint32_t at = cols == 64 ? tile_at<64>(rr, pp) : tile_at<DK>(rr, pp);
                *reinterpret_cast<uint32_t*>(tile + at + c4 * 4) = w[i];
            }
        };
        auto stage_tok = [&](size_t off, size_t off_inv, int terms, float most, char* dst, int sl0) {
#pragma unroll
            for (int q = 0; q < SL * 4 * KT * 32 / 512; ++q) {  // (term, slice, chunk, kk), a warp each
                const int i = warp + 16 * q, kk = i & 1, ch = (i >> 1) & 1, sl = (i >> 2) % SL, term = (i >> 2) / SL;
                uint4 x = make_uint4(0, 0, 0, 0);
                float ratio = 1.0f;
                if (sl0 + sl < a.l.slices && ch < nchunks) {
                    const size_t at = ((size_t)n * a.l.nch + 2 * blk + ch) * a.l.slices + sl0 + sl;
                    x = reinterpret_cast<const uint4*>(a.ws + off)[(at * terms + term) * 64 + kk * 32 + lane];
                    ratio = reinterpret_cast<const float*>(a.ws + off_inv)[at] / most;
                }
                put(dst + term * TT, 64, sl * 16 + g, (ch * 2 + kk) * 2, x, ratio);
            }
        };
        auto stage_state = [&](size_t off, size_t off_lo, int terms, size_t off_inv, float most, int sl0) {
#pragma unroll
            for (int q = 0; q < SL * KT * (DK / 16) / 16; ++q) {
                const int i = warp + 16 * q, kk = i % (DK / 16), sl = i / (DK / 16) % SL, term = i / (DK / 16) / SL;
                uint4 x = make_uint4(0, 0, 0, 0);
                float ratio = 1.0f;
                if (sl0 + sl < a.l.slices) {
                    const size_t at = ((size_t)n * (a.l.nblk + 1) + blk) * a.l.slices + sl0 + sl;
                    const char* src = off_lo ? a.ws + (term ? off_lo : off) + at * a.l.state_bytes : a.ws + off + (at * terms + term) * a.l.state_bytes;
                    x = reinterpret_cast<const uint4*>(src)[kk * 32 + lane];
                    ratio = reinterpret_cast<const float*>(a.ws + off_inv)[at] / most;
                }
                put(st_s + term * TS, DK, sl * 16 + g, kk * 2, x, ratio);
            }
        };
        auto stage_do = [&](int d0) {  // [64 tokens][ROWS value rows]
#pragma unroll
            for (int q = 0; q < 64 * ROWS / 8 / 512 + (64 * ROWS / 8 < 512); ++q) {
                const int i = tid + 512 * q, row = i / (ROWS / 8), piece = i % (ROWS / 8), t = t0 + row, d = d0 + piece * 8;
                if (row >= 64) continue;
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = 0.0f;
                if (t < s.L && d < s.dv) {
                    const IO* p = reinterpret_cast<const IO*>(ba.d_o) + ((size_t)n * s.L + t) * s.dv + d;
                    if (vec && sizeof(IO) == 2) {
                        const uint4 raw = *reinterpret_cast<const uint4*>(p);
                        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (d + j < s.dv) x[j] = to_f32(p[j]);
                    }
                }
                uint4 hi, lo;
                split(x[0] * so, x[1] * so, hi.x, lo.x); split(x[2] * so, x[3] * so, hi.y, lo.y);
                split(x[4] * so, x[5] * so, hi.z, lo.z); split(x[6] * so, x[7] * so, hi.w, lo.w);
                const uint32_t at = tile_at<ROWS>(row, piece);
                *reinterpret_cast<uint4*>(st_o + at) = hi;
                if (KT == 2) *reinterpret_cast<uint4*>(st_o + TT + at) = lo;
            }
        };
        // two terms each, without the product of the second ones
        auto product = [&](float (&c)[4], const uint32_t (&x)[KT][4], const uint32_t (&b)[KT][4], int y) {
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int u = 0; u + t < KT; ++u) mma(c, x[t], b[u][2 * y], b[u][2 * y + 1]);
        };
        float sg[2][4] = {}, kp[2][4] = {}, aq[NT][4] = {}, ak[NT][4] = {};
        for (int sl0 = 0; sl0 < a.l.slices; sl0 += SL) {
            stage_state(a.l.S, KT == 2 ? a.l.S_lo : 0, 1, a.l.s_inv, iS, sl0);
            stage_tok(a.l.e, a.l.e_inv, 2, iu, st_u, sl0);
            stage_tok(a.l.dp, a.l.dp_inv, KT, ip, st_p, sl0);
            stage_do(sl0 * 16);
            __syncthreads();
            const int steps = min(SL, a.l.slices - sl0);
#pragma unroll 2
            for (int kk = 0; kk < steps; ++kk) {
                uint32_t ao[KT][4], ap[KT][4], b[KT][4];
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    ldsm4(ao[t], addr_mk<ROWS>(os + t * TT, tw * 16, kk, lane));
                    ldsm4_t(ap[t], addr_km<64>(ps + t * TT, tw * 16, kk, lane));
                }
                if (hw <= tw) {  // not the tokens after these
#pragma unroll
                    for (int t = 0; t < KT; ++t) ldsm4_t(b[t], addr_kn<64>(us + t * TT, hw * 2, kk, lane));
                    product(sg[0], ao, b, 0); product(sg[1], ao, b, 1);
                    product(kp[0], ap, b, 0); product(kp[1], ap, b, 1);
                }
#pragma unroll
                for (int h = 0; h < NT / 2; ++h) {
#pragma unroll
                    for (int t = 0; t < KT; ++t) ldsm4_t(b[t], addr_kn<DK>(ss + t * TS, hw * NT + 2 * h, kk, lane));
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        product(aq[2 * h + y], ao, b, y);
                        product(ak[2 * h + y], ap, b, y);
                    }
                }
            }
            __syncthreads();
        }
        {
            const float q0 = s.scale * bt[row0], q1 = s.scale * bt[row1], k0 = -bt[row0], k1 = -bt[row1];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                tq[j][0] = fmaf(aq[j][0] * (io * iS), q0, tq[j][0]); tq[j][1] = fmaf(aq[j][1] * (io * iS), q0, tq[j][1]);
                tq[j][2] = fmaf(aq[j][2] * (io * iS), q1, tq[j][2]); tq[j][3] = fmaf(aq[j][3] * (io * iS), q1, tq[j][3]);
                tk[j][0] = fmaf(ak[j][0] * (ip * iS), k0, tk[j][0]); tk[j][1] = fmaf(ak[j][1] * (ip * iS), k0, tk[j][1]);
                tk[j][2] = fmaf(ak[j][2] * (ip * iS), k1, tk[j][2]); tk[j][3] = fmaf(ak[j][3] * (ip * iS), k1, tk[j][3]);
#pragma unroll
                for (int x = 0; x < 4; ++x) aq[j][x] = ak[j][x] = 0.0f;
            }
        }
        // D and eta on both token-by-token matrices, their largest magnitudes
        float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int t = x < 2 ? row0 : row1, u = hw * 16 + j * 8 + 2 * c4 + (x & 1);
                const float D = u <= t ? expf((float)(run[t] - run[u])) * eta[u] : 0.0f;
                sg[j][x] = u <= t ? sg[j][x] * (io * iu) * (D * s.scale) : 0.0f;
                kp[j][x] = u < t ? -kp[j][x] * (ip * iu) * D : 0.0f;
                m0 = fmaxf(m0, fabsf(sg[j][x]));
                m1 = fmaxf(m1, fabsf(kp[j][x]));
            }
        m0 = warp_max(m0); m1 = warp_max(m1);
        if (lane == 0) { red[warp] = m0; red[16 + warp] = m1; }
        if (a.l.slices <= SL) stage_state(a.l.X, 0, KT, a.l.x_inv, iX, 0);  // everything has been read
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) { m0 = fmaxf(m0, red[i]); m1 = fmaxf(m1, red[16 + i]); }
        float fs, gs, fk, gk;
        pow2_scale(m0, fs, gs);
        pow2_scale(m1, fk, gk);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int t = x ? row1 : row0, u = hw * 16 + j * 8 + 2 * c4;
                uint32_t w[2];
                split(sg[j][2 * x] * fs, sg[j][2 * x + 1] * fs, w[0], w[1]);
                const uint32_t at = tile_at<64>(t, u >> 3) + (u & 7) * 2;
                char* kap = mat + KT * 8192;
#pragma unroll
                for (int term = 0; term < KT; ++term) *reinterpret_cast<uint32_t*>(mat + term * 8192 + at) = w[term];
                split(kp[j][2 * x] * fk, kp[j][2 * x + 1] * fk, w[0], w[1]);
                // kappa + kappa^T: the strictly lower half, its mirror image and a zero diagonal
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t mt = tile_at<64>(u + y, t >> 3) + (t & 7) * 2;
#pragma unroll
                    for (int term = 0; term < KT; ++term) {
                        const uint16_t z = (uint16_t)(w[term] >> (16 * y));
                        if (u + y <= t) *reinterpret_cast<uint16_t*>(kap + term * 8192 + at + 2 * y) = z;
                        if (u + y < t) *reinterpret_cast<uint16_t*>(kap + term * 8192 + mt) = z;
                    }
                }
            }
        // eta D_end X^T e
        for (int sl0 = 0; sl0 < a.l.slices; sl0 += SL) {
            if (a.l.slices > SL) {
                stage_tok(a.l.e, a.l.e_inv, 2, iu, st_u, sl0);
                stage_state(a.l.X, 0, KT, a.l.x_inv, iX, sl0);
            }
            __syncthreads();
            const int steps = min(SL, a.l.slices - sl0);
#pragma unroll 2
            for (int kk = 0; kk < steps; ++kk) {
                uint32_t au[KT][4], b[KT][4];
#pragma unroll
                for (int t = 0; t < KT; ++t) ldsm4_t(au[t], addr_km<64>(us + t * TT, tw * 16, kk, lane));
#pragma unroll
                for (int h = 0; h < NT / 2; ++h) {
#pragma unroll
                    for (int t = 0; t < KT; ++t) ldsm4_t(b[t], addr_kn<DK>(ss + t * TS, hw * NT + 2 * h, kk, lane));
#pragma unroll
                    for (int y = 0; y < 2; ++y) product(ak[2 * h + y], au, b, y);
                }
            }
            if (a.l.slices > SL) __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const float f0 = dend[row0], f1 = dend[row1];
            tk[j][0] = fmaf(ak[j][0] * (iu * iX), f0, tk[j][0]); tk[j][1] = fmaf(ak[j][1] * (iu * iX), f0, tk[j][1]);
            tk[j][2] = fmaf(ak[j][2] * (iu * iX), f1, tk[j][2]); tk[j][3] = fmaf(ak[j][3] * (iu * iX), f1, tk[j][3]);
#pragma unroll
            for (int x = 0; x < 4; ++x) ak[j][x] = 0.0f;
        }
        // sigma K, sigma^T Q, (kappa + kappa^T) K: three sums with scales of their own
        auto times = [&](float (&acc)[NT][4], uint32_t rows, uint32_t tile, bool transposed, int k0, int k1) {
#pragma unroll 2
            for (int kk = k0; kk < k1; ++kk) {
                uint32_t x[KT][4], b[KT][4];
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    if (transposed) ldsm4_t(x[t], addr_km<64>(rows + t * 8192, tw * 16, kk, lane));
                    else ldsm4(x[t], addr_mk<64>(rows + t * 8192, tw * 16, kk, lane));
                }
#pragma unroll
                for (int h = 0; h < NT / 2; ++h) {
#pragma unroll
                    for (int t = 0; t < KT; ++t) ldsm4_t(b[t], addr_kn<DK>(tile + t * 128 * DK, hw * NT + 2 * h, kk, lane));
#pragma unroll
                    for (int y = 0; y < 2; ++y) product(acc[2 * h + y], x, b, y);
                }
            }
        };
        times(aq, ms, ks, false, 0, tw + 1);
        times(ak, ms, qs, true, tw, 4);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                tq[j][x] = fmaf(aq[j][x], gs * ik, tq[j][x]);
                tk[j][x] = fmaf(ak[j][x], gs * iq, tk[j][x]);
                ak[j][x] = 0.0f;
            }
        times(ak, ms + KT * 8192, ks, false, 0, 4);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) tk[j][x] = fmaf(ak[j][x], gk * ik, tk[j][x]);
    }
    IO* dq = reinterpret_cast<IO*>(ba.dq) + (size_t)nk * s.L * s.dk;
    IO* dk = reinterpret_cast<IO*>(ba.dk) + (size_t)nk * s.L * s.dk;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int t = t0 + (x < 2 ? row0 : row1), col = (hw * NT + j) * 8 + 2 * c4 + (x & 1);
            if (t < s.L && col < s.dk) {
                dq[(size_t)t * s.dk + col] = from_f32<IO>(tq[j][x]);
                dk[(size_t)t * s.dk + col] = from_f32<IO>(tk[j][x]);
            }
        }
}

template <typename IO, int DK, int KT> int launch(const DeltaBwdArgs& b, cudaStream_t st) {
    const DeltaArgs& a = b.f;
    {
        constexpr int bytes = kStages * stage_bytes<DK, KT>();
        auto kernel = delta_chain_kernel<IO, DK, KT>;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return (int)e;
        int w = 4;
        while (w > 1 && a.l.N * ((a.l.slices + w - 1) / w) < 96) w >>= 1;
        kernel<<<(unsigned)(a.l.N * ((a.l.slices + w - 1) / w)), w * 32, bytes, st>>>(b, w);
        e = cudaGetLastError();
        if (e != cudaSuccess) return (int)e;
    }
    {
        constexpr int bytes = qk_smem<DK, KT>();
        static_assert(bytes <= 227 * 1024, "shared memory of the dq / dk kernel");
        auto kernel = delta_qk_kernel<IO, DK, KT>;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return (int)e;
        const bool vec = a.s.dv % 8 == 0 && reinterpret_cast<uintptr_t>(b.d_o) % 16 == 0;
        kernel<<<(unsigned)(a.l.Nk * a.l.nblk), 512, bytes, st>>>(b, vec);
        e = cudaGetLastError();
        if (e != cudaSuccess) return (int)e;
    }
    delta_gate_kernel<<<(unsigned)(a.l.N * a.l.nsup), kDeltaSuper * 64, 0, st>>>(b);
    return (int)cudaGetLastError();
}

}  // namespace

int delta_bwd_launch(const DeltaBwdArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.f.s.f32) return a.f.l.DK == 64 ? launch<float, 64, 2>(a, st) : launch<float, 128, 2>(a, st);
    return a.f.l.DK == 64 ? launch<__nv_bfloat16, 64, 1>(a, st) : launch<__nv_bfloat16, 128, 1>(a, st);
}

}  // namespace e2ttt
