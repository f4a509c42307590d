// Gated delta rule, reverse pass.  With X the adjoint of the state behind a chunk and Z = (I + eta strict(D K K^T))^-T dU:
//   dU = A^T dO + D_end X K,   dP = eta Z = dV,   X_before = b_end X + scale (b dO) Q^T - (b dP) K^T            (delta_chain_kernel)
//   dQ = (D dO^T U) K + scale b S_0^T dO,   dK = (D dO^T U)^T Q - (W + W^T) K - b S_0^T dP + D_end X^T U,  W = strict(D dP^T U)   (delta_qk_kernel)
//   d eta = Z . e,   d log_gamma_t = <X'_t, g_t S_{t-1}>: what tokens before t hand on to tokens from t on, over a chunk                (delta_gate_kernel)
//     = sum_{i < t <= s} eta_i (A_si dO_s . e_i - (D K K^T)_si dP_s . e_i) + sum_{s >= t} b_s (scale dO_s . S_0 q_s - dP_s . S_0 k_s)
//       + sum_{i < t} eta_i D_end,i e_i . X k_i + b_end <X, S_0>,   X'_t the adjoint with what token t reads.
// Every term carries the decays between its two ends as factors, so a token that forgets the state has an exact small gradient: sums of
// outputs and values (o_s . do_s - v_s . dv_s and so on) would have to cancel to it.  The walks have S_0 Q^T, S_0 K^T and X K^T at hand.
// The chain walks the chunks from the last to the first as the forward does, a warp per 16 value rows; dQ and dK contract over the
// value rows of all warps and are left to a kernel that takes the blocks side by side.
#include "api_checks.h"
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

constexpr int kStages = 3;
constexpr int kGateWarps = 4;

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

// what the warps of a slice hand over, a buffer per parity of the step: from the side warp A^T dO, the fragments of b dO and bounds on both; from the
// chain Z, X's fragments behind a block (first term, with fp32 I/O both); and what the side warp has fetched
template <int DK, int KT, int KS> struct alignas(128) ReverseExchange {
    uint4 x[KT][DK / 16][32];
    uint4 q[2][2][32];        // [term][k-step]
    float4 in[4][32], z[4][32];
    float4 part[KS > 1 ? KS : 1][4][KS > 1 ? 32 : 1];
    uint4 e[2][2][32];        // e's fragments
    float4 sq[4][32];         // S Q^T of the forward
    float4 sk[4][32];                            // S K^T of the forward
    float4 xk[KS > 1 ? 4 : 1][KS > 1 ? 32 : 1];  // X K^T; with one warp it takes the place of `in`, which the same lane has read
    float4 d_o[KT == 1 ? 2 : 4][32];
    uint4 out[KT == 1 ? 64 : 1];
    float norm[KS];
    float x_inv, in_max, q_max, q_inv, q_sum;
};
template <int DK, int KT, int KS> constexpr int chain_smem(int slices) {
    return kStages * stage_bytes<DK, KT>() + 2 * slices * (int)sizeof(ReverseExchange<DK, KT, KS>);
}

// The chain X, Z, X runs as the forward's does (a warp per slice, or KS by columns; scales from bounds; the products of a chunk between the steps of
// its arithmetic).  A side warp per slice, a chunk ahead, makes what does not depend on X (A^T dO, the fragments of b dO, o . dO), and, a chunk
// behind, what hangs off Z (dV, dP's fragments, the sums for d eta and d log_gamma).  Bound by what a chunk's steps issue one after the other:
// 4 x 16 sequences of 4096 tokens, 128 x 128, bf16, in 423 us (3.3 us a chunk); 8 x 12 of 2048 tokens, 64 x 64, in 162 us.
template <typename IO, int DK, int KT, int KS>
__global__ void __launch_bounds__(KS == 1 ? 256 : 160, 1) delta_chain_kernel(const DeltaBwdArgs ba, const int per, const bool vec) {
    extern __shared__ __align__(1024) char smem[];
    constexpr int NS = kStages, DC = DK / KS, SB = stage_bytes<DK, KT>(), TERMS = KT == 2 ? 3 : 2;
    __shared__ uint64_t full[NS];
    __shared__ int dead_flag;
    using X = ReverseExchange<DK, KT, KS>;
    const DeltaArgs& a = ba.f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const DeltaShape& s = a.s;
    const int groups = (a.l.slices + per - 1) / per;
    const int64_t n = blockIdx.x / groups, nk = (n / s.H) * s.Hk + (n % s.H) / (s.H / s.Hk);
    const bool chain = warp < per * KS;
    const int mine = chain ? warp / KS : warp - per * KS, part = chain ? warp % KS : 0;
    const int slice = (int)(blockIdx.x % groups) * per + mine;
    const bool active = slice < a.l.slices;
    const int nch = a.l.nch;
    X* xb = reinterpret_cast<X*>(smem + NS * SB) + 2 * mine;
    sm100::WaitCtx wait{&dead_flag, reinterpret_cast<int*>(a.ws)};
    if (threadIdx.x == 0) {
        for (int i = 0; i < NS; ++i) sm100::mbar_init(&full[i], 1);
        dead_flag = 0;
        sm100::fence_mbar_init();
    }
    __syncthreads();
    const int r0 = slice * 16 + g, r1 = r0 + 8;
    const bool ok0 = active && r0 < s.dv, ok1 = active && r1 < s.dv;
    const uint32_t ring = sm100::smem_u32(smem);
    // a stage: K, Q, then the record's scalars, A, T
    constexpr int AT_SC = 2 * KT * 64 * DK, AT_A = AT_SC + 1024, AT_T = AT_A + 4096;

    if (chain) {
        const int col0 = part * DC;
        float S[DC / 8][4], s_now = 1.0f, s_inv = 1.0f, norm = 0.0f;  // X times its scale
#pragma unroll
        for (int j = 0; j < DC / 8; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int col = col0 + j * 8 + 2 * c4 + (x & 1);
                const bool ok = ba.dS_final && col < s.dk && (x < 2 ? ok0 : ok1);
                S[j][x] = ok ? ba.dS_final[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] : 0.0f;
            }
        // |dU| <= max |A^T dO| + max D_end |k| |X|,  |Z| <= column sums of |T| |dU|,  |X_before| <= b_end |X| + max |dO| sum b |q| + |Z| sum |eta| b |k|
        float sk[4][4], squares0 = 0.0f, squares1 = 0.0f;  // X K^T of the next chunk
        uint32_t fh[2][4], fl[2][4];
        auto split_s = [&](int kk, int r) {
            const float (&y)[4] = S[2 * kk + (r >> 1)];
            const float y0 = y[2 * (r & 1)], y1 = y[2 * (r & 1) + 1];
            fma2(squares0, squares1, y0, y1, y0, y1, squares0, squares1);
            split(y0, y1, fh[kk & 1][r], fl[kk & 1][r]);
        };
        auto leave_s = [&](int kk, X& x) {
            const uint32_t (&h)[4] = fh[kk & 1], (&l)[4] = fl[kk & 1];
            x.x[0][part * (DC / 16) + kk][lane] = make_uint4(h[0], h[1], h[2], h[3]);
            if (KT == 2) x.x[KT - 1][part * (DC / 16) + kk][lane] = make_uint4(l[0], l[1], l[2], l[3]);
        };
        auto times_k = [&](int kk, int i, bool first, const uint32_t (&b)[2 * KT][4]) {
            const int term = i >> 1, h = i & 1;
            const uint32_t (&x)[4] = term == 1 ? fl[kk & 1] : fh[kk & 1];
            const uint32_t (&y)[4] = b[term == 2 ? 2 * KT - 2 + h : h];
            if (first && term == 0) {
                mma0(sk[2 * h], x, y[0], y[1]);
                mma0(sk[2 * h + 1], x, y[2], y[3]);
            } else {
                mma(sk[2 * h], x, y[0], y[1]);
                mma(sk[2 * h + 1], x, y[2], y[3]);
            }
        };
        auto load_k = [&](uint32_t ks, int kk, uint32_t (&b)[2 * KT][4]) {
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                ldsm4(b[2 * t], addr_nk<DK>(ks + t * 64 * DK, 0, part * (DC / 16) + kk, lane));
                ldsm4(b[2 * t + 1], addr_nk<DK>(ks + t * 64 * DK, 2, part * (DC / 16) + kk, lane));
            }
        };
        auto hand = [&](X& x) {
            const float y = 32.0f * warp_most(squares0 + squares1);
            if (KS == 1) {
                norm = y;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x.part[part][j][lane] = make_float4(sk[j][0], sk[j][1], sk[j][2], sk[j][3]);
                if (lane == 0) x.norm[part] = y;
            }
            if (lane == 0 && part == 0) x.x_inv = s_inv;
        };
        auto take = [&](const X& x) {
            if (KS > 1) {
                norm = 0.0f;
#pragma unroll
                for (int h = 0; h < KS; ++h) {
                    norm += x.norm[h];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 z = x.part[KS > 1 ? h : 0][j][lane];
                        if (h == 0) { sk[j][0] = z.x; sk[j][1] = z.y; sk[j][2] = z.z; sk[j][3] = z.w; }
                        else { sk[j][0] += z.x; sk[j][1] += z.y; sk[j][2] += z.z; sk[j][3] += z.w; }
                    }
                }
            }
            float root;
            asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(norm));
            norm = root * s_inv;
        };
        wait_phase(&full[0], 0, wait, 902);
        if (active) {
            float m = 0.0f;
            for (int col = c4; col < s.dk && ba.dS_final; col += 4) {
                if (ok0) m = fmaxf(m, fabsf(ba.dS_final[((size_t)n * s.dv + r0) * s.dk + col]));
                if (ok1) m = fmaxf(m, fabsf(ba.dS_final[((size_t)n * s.dv + r1) * s.dk + col]));
            }
            pow2_bound(warp_max(m), s_now, s_inv);
#pragma unroll
            for (int j = 0; j < DC / 8; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) S[j][x] *= s_now;
#pragma unroll
            for (int kk = 0; kk < DC / 16; ++kk) {
                uint32_t b[2 * KT][4];
                load_k(ring, kk, b);
#pragma unroll
                for (int r = 0; r < 4; ++r) split_s(kk, r);
                leave_s(kk, xb[0]);
#pragma unroll
                for (int i = 0; i < 2 * TERMS; ++i) times_k(kk, i, kk == 0, b);
            }
            hand(xb[0]);
            sm100::fence_proxy_async_smem();  // X behind the last chunk is copied from there
        }
        __syncthreads();  // the side warp's part of the last chunk
        int st = 0, st_next = 1, phase_next = 0;
        for (int i = 0; i < nch; ++i) {
            const int c = nch - 1 - i;
            const uint32_t ks = ring + st * SB, qs = ks + KT * 64 * DK, ts = ks + AT_T, kn = ring + st_next * SB;
            const float* sc = reinterpret_cast<const float*>(smem + st * SB + AT_SC);
            const float* head = sc + kRecHead * 32;
            X& x = xb[i & 1];
            X& xn = xb[(i + 1) & 1];
            float w_old = 0.0f, w_new = 0.0f;
            uint32_t wh[2][4], wl[2][4], qh[2][4], ql[2][4];
            const bool come = i + 1 == nch || probe_phase(&full[st_next], phase_next);
            if (active) {
                take(x);
                if (!(c & 1)) {  // <X, S>: behind a block's first chunk, before it
                    const size_t at = ((size_t)n * a.l.nblk + (c >> 1)) * a.l.slices + slice;
                    const uint4* hi4 = reinterpret_cast<const uint4*>(a.ws + a.l.S + at * a.l.state_bytes) + part * (DC / 16) * 32 + lane;
                    const uint4* lo4 = reinterpret_cast<const uint4*>(a.ws + a.l.S_lo + at * a.l.state_bytes) + part * (DC / 16) * 32 + lane;
                    float h = 0.0f;
#pragma unroll
                    for (int kk = 0; kk < DC / 16; ++kk) {
                        const uint4 u = hi4[kk * 32], v2 = lo4[kk * 32];
                        const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v2.x, v2.y, v2.z, v2.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float y0, y1;
                            join_terms(uw[r], vw[r], y0, y1);
                            const float (&y)[4] = S[2 * kk + (r >> 1)];
                            h = fmaf(y[2 * (r & 1)], y0, h);
                            h = fmaf(y[2 * (r & 1) + 1], y1, h);
                        }
                    }
                    h = warp_sum(h) * (s_inv * reinterpret_cast<const float*>(a.ws + a.l.s_inv)[at]);
                    float* hx = reinterpret_cast<float*>(a.ws + a.l.hx) + at * 4;
                    if (lane == 0) hx[part] = h;
                    if (lane >= KS && lane < 4 && part == 0) hx[lane] = 0.0f;
                }
                uint32_t th[3][4], tl[3][4];  // (tokens 0-15 x 0-15), (16-31 x 0-15), (16-31 x 16-31)
                ldsm4_t(th[0], addr_kn<32>(ts, 0, 0, lane)); ldsm4_t(th[1], addr_kn<32>(ts, 0, 1, lane)); ldsm4_t(th[2], addr_kn<32>(ts, 2, 1, lane));
                ldsm4_t(tl[0], addr_kn<32>(ts + 2048, 0, 0, lane)); ldsm4_t(tl[1], addr_kn<32>(ts + 2048, 0, 1, lane));
                ldsm4_t(tl[2], addr_kn<32>(ts + 2048, 2, 1, lane));
                const float bend = head[kHeadEnd];
                const float ub = fmaf(head[kHeadKe], norm, x.in_max), zb = ub * head[kHeadRsum];
                float f, q;
                pow2_bound(ub, f, q);
                // dU, times its scale f
                float p[4][4], z[4][4];
                const float fs = scales(f, s_inv);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 in = x.in[j][lane];
                    if (KS == 1) x.in[j][lane] = make_float4(sk[j][0], sk[j][1], sk[j][2], sk[j][3]);
                    else if (part == (j >> 1)) x.xk[KS > 1 ? j : 0][KS > 1 ? lane : 0] = make_float4(sk[j][0], sk[j][1], sk[j][2], sk[j][3]);
                    const float2 de = *reinterpret_cast<const float2*>(sc + kRecDend * 32 + j * 8 + 2 * c4);
                    float y0, y1;
                    mul2(y0, y1, de.x, de.y, fs, fs);
                    mul2(p[j][0], p[j][1], in.x, in.y, f, f);
                    mul2(p[j][2], p[j][3], in.z, in.w, f, f);
                    fma2(p[j][0], p[j][1], sk[j][0], sk[j][1], y0, y1, p[j][0], p[j][1]);
                    fma2(p[j][2], p[j][3], sk[j][2], sk[j][3], y0, y1, p[j][2], p[j][3]);
                }
                {
                    uint32_t h0[4], l0[4], h1[4], l1[4];
                    split_a(p[2], p[3], h1, l1);
                    mma0(z[0], h1, th[1][0], th[1][1]); mma0(z[1], h1, th[1][2], th[1][3]);
                    mma0(z[2], h1, th[2][0], th[2][1]); mma0(z[3], h1, th[2][2], th[2][3]);
                    split_a(p[0], p[1], h0, l0);
                    float t[4][4];  // the second terms' products apart
                    mma0(t[0], l1, th[1][0], th[1][1]); mma0(t[1], l1, th[1][2], th[1][3]);
                    mma0(t[2], l1, th[2][0], th[2][1]); mma0(t[3], l1, th[2][2], th[2][3]);
                    mma(z[0], h0, th[0][0], th[0][1]); mma(z[1], h0, th[0][2], th[0][3]);
                    mma(t[0], h1, tl[1][0], tl[1][1]); mma(t[1], h1, tl[1][2], tl[1][3]);
                    mma(t[2], h1, tl[2][0], tl[2][1]); mma(t[3], h1, tl[2][2], tl[2][3]);
                    mma(t[0], l0, th[0][0], th[0][1]); mma(t[1], l0, th[0][2], th[0][3]);
                    mma(t[0], h0, tl[0][0], tl[0][1]); mma(t[1], h0, tl[0][2], tl[0][3]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        add2(z[j][0], z[j][1], t[j][0], t[j][1]);
                        add2(z[j][2], z[j][3], t[j][2], t[j][3]);
                    }
                }
                // z times qe is Z.  - eta b Z and b dO go into the state at one scale, fw: the fragments of b dO, which are there at their own, move to it
                const float qe = q * head[kHeadR];
                float fw, w_inv;
                pow2_bound(fmaxf(zb * head[kHeadZmax], x.q_max), fw, w_inv);
                const float ratio = fw * x.q_inv;
                const __half2 move = __float2half2_rn(ratio);
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const uint4 h4 = x.q[0][kk][lane], l4 = x.q[1][kk][lane];
                    const uint32_t hw[4] = {h4.x, h4.y, h4.z, h4.w}, lw[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&hw[r]), move), y2 = __hmul2(*reinterpret_cast<const __half2*>(&lw[r]), move);
                        qh[kk][r] = *reinterpret_cast<const uint32_t*>(&y);
                        ql[kk][r] = *reinterpret_cast<const uint32_t*>(&y2);
                    }
                }
                if (ratio < 0x1p-14f) {  // dO far below the adjoint: what of it fits this scale, where the ratio itself has few bits in fp16 or none
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        const uint4 h4 = x.q[0][kk][lane], l4 = x.q[1][kk][lane];
                        const uint32_t hw[4] = {h4.x, h4.y, h4.z, h4.w}, lw[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float y0, y1;
                            join_terms(hw[r], lw[r], y0, y1);
                            split(y0 * ratio, y1 * ratio, qh[kk][r], ql[kk][r]);
                        }
                    }
                }
                const float wf = -scales(fw, qe), old_inv = s_inv;
                pow2_bound(fmaf(bend, norm, fmaf(zb, head[kHeadZsum], x.q_sum)), s_now, s_inv);
                w_old = scales(bend * old_inv, s_now);
                w_new = w_inv * s_now;
                float w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 ze = *reinterpret_cast<const float2*>(sc + kRecZ * 32 + j * 8 + 2 * c4);
                    float y0, y1;
                    mul2(y0, y1, ze.x, ze.y, wf, wf);
                    mul2(w[j][0], w[j][1], z[j][0], z[j][1], y0, y1);
                    mul2(w[j][2], w[j][3], z[j][2], z[j][3], y0, y1);
                    if (KS == 1 || part == (j >> 1)) {
                        float4 t;
                        mul2(t.x, t.y, z[j][0], z[j][1], qe, qe);
                        mul2(t.z, t.w, z[j][2], z[j][3], qe, qe);
                        x.z[j][lane] = t;
                    }
                }
                split_a(w[0], w[1], wh[0], wl[0]);
                split_a(w[2], w[3], wh[1], wl[1]);
            }
            if (!come) sm100::mbar_wait(&full[st_next], phase_next, wait, 902);
            if (active) {
                constexpr int NJ = DC / 32;
                float y[2][4][4];
                uint32_t fs[2][2][KT][4], fk[2][2 * KT][4];
                auto load_s = [&](uint32_t tile, int j4) {
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int k = 0; k < KT; ++k) ldsm4_t(fs[kk][h][k], addr_kn<DK>(tile + k * 64 * DK, part * (DC / 8) + 4 * j4 + 2 * h, kk, lane));
                };
                // the i-th two MMAs: 4 TERMS with the keys, then as many with the queries
                auto sum = [&](float (&t)[4][4], int i) {
                    const bool keys = i < 4 * TERMS;
                    const int m = keys ? i : i - 4 * TERMS, kk = m / (2 * TERMS), term = m % (2 * TERMS) >> 1, h = m & 1;
                    const uint32_t (&w)[4] = keys ? (term == 1 ? wl[kk] : wh[kk]) : (term == 1 ? ql[kk] : qh[kk]);
                    const uint32_t (&b)[4] = fs[kk][h][term == 2 ? KT - 1 : 0];
                    if (i < 2) {
                        mma0(t[2 * h], w, b[0], b[1]);
                        mma0(t[2 * h + 1], w, b[2], b[3]);
                    } else {
                        mma(t[2 * h], w, b[0], b[1]);
                        mma(t[2 * h + 1], w, b[2], b[3]);
                    }
                };
                load_s(ks, 0);
                squares0 = squares1 = 0.0f;
#pragma unroll
                for (int m = 0; m < 4 * TERMS; ++m) sum(y[0], m);
                load_s(qs, 0);
                load_k(kn, 0, fk[0]);
#pragma unroll
                for (int m = 4 * TERMS; m < 8 * TERMS; ++m) sum(y[0], m);
                if (NJ > 1) load_s(ks, 1);
                const bool kept = c & 1 ? false : c > 0;  // X before this chunk is X behind a block
#pragma unroll
                for (int j4 = 0; j4 < NJ; ++j4) {
                    const int before = j4 > 0 ? 2 * TERMS : 0, next = j4 + 1 < NJ ? 8 * TERMS : 0, all = before + next + 2 * TERMS;
                    auto upto = [&](int m) {
                        const int most = m < 5 ? before + next : all;
                        return (m + 1) * all / 12 < most ? (m + 1) * all / 12 : most;
                    };
                    auto issue = [&](int m) {
                        if (m < before) times_k(2 * j4 - 1, m, false, fk[1]);
                        else if (m < before + next) sum(y[(j4 + 1) & 1], m - before);
                        else times_k(2 * j4, m - before - next, j4 == 0, fk[0]);
                        if (m + 1 == before || (m == 0 && before == 0)) load_k(kn, 2 * j4 + 1, fk[1]);
                        if (next > 0 && m + 1 == before + next / 2) load_s(qs, j4 + 1);
                        if (next > 0 && m + 1 == before + next && j4 + 2 < NJ) load_s(ks, j4 + 2);
                    };
#pragma unroll
                    for (int m = 0; m < 12; ++m) {
                        if (m == 0 || m == 1 || m == 6 || m == 7) {
                            const int k = m < 2 ? m : m - 4;
                            float (&d)[4] = S[4 * j4 + k];
                            const float (&t)[4] = y[j4 & 1][k];
#pragma unroll
                            for (int z = 0; z < 4; z += 2) {
                                float m0, m1;
                                mul2(m0, m1, d[z], d[z + 1], w_old, w_old);
                                fma2(d[z], d[z + 1], t[z], t[z + 1], w_new, w_new, m0, m1);
                            }
                        } else {
                            const int r = m < 6 ? m - 2 : m - 8;
                            split_s(2 * j4 + (m < 6 ? 0 : 1), r);
                            if (r == 3 && kept) leave_s(2 * j4 + (m < 6 ? 0 : 1), xn);
                        }
#pragma unroll
                        for (int k = 0; k < 2 * TERMS; ++k)
                            if (upto(m - 1) + k < upto(m)) issue(upto(m - 1) + k);
                    }
                    if (j4 + 1 < NJ) load_k(kn, 2 * j4 + 2, fk[0]);
                }
#pragma unroll
                for (int k = 0; k < 2 * TERMS; ++k) times_k(2 * NJ - 1, k, false, fk[1]);
                hand(xn);
                if (kept) sm100::fence_proxy_async_smem();
            }
            st = st_next;
            if (++st_next == NS) { st_next = 0; phase_next ^= 1; }
            __syncthreads();
        }
        if (active) {
#pragma unroll
            for (int j = 0; j < DC / 8; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int col = col0 + j * 8 + 2 * c4 + (x & 1);
                    if (col < s.dk && (x < 2 ? ok0 : ok1)) ba.dS_init[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] = S[j][x] * s_inv;
                }
        }
        return;
    }

    // ---- the side warp of a slice; step i is chunk nch - 1 - i
    const char* qk_src = a.ws + a.l.qk + (size_t)nk * nch * a.l.qk_bytes;
    const char* rec_src = a.ws + a.l.rec + (size_t)n * nch * a.l.rec_bytes + kDeltaRecSkip;
    const bool fetches = mine == 0 && lane == 0;
    auto fetch = [&](int i, int st) {
        const int c = nch - 1 - i;
        const uint32_t dst = ring + st * SB;
        uint64_t* bar = &full[st];
        sm100::mbar_expect_tx(bar, SB);
        bulk_copy(dst, qk_src + (size_t)c * a.l.qk_bytes, 2 * KT * 64 * DK, bar);
        bulk_copy(dst + 2 * KT * 64 * DK, rec_src + (size_t)c * a.l.rec_bytes, kDeltaRecBytes, bar);
    };
    if (fetches)
        for (int i = 0; i < NS && i < nch; ++i) fetch(i, i);
    __syncwarp();
    const int rows = active ? min(16, s.dv - slice * 16) : 0;
    const size_t seq = (size_t)n * s.L * s.dv + slice * 16;
    const IO* d_o = reinterpret_cast<const IO*>(ba.d_o) + seq;
    IO* dv = reinterpret_cast<IO*>(ba.dv) + seq;
    auto copy16 = [&](const void* dst, const void* src, int bytes) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sm100::smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
    };
    // a chunk's rows of dO to a tile of tokens (bf16) or to fragment order (fp32)
    auto load_tok = [&](float4* dst, const IO* src, int c) {
        if (KT == 1) {
            const int t = c * kDeltaChunk + lane;
            const IO* p = src + (size_t)t * s.dv;
            const int here = t < s.L ? rows : 0;
            if (vec) {
#pragma unroll
                for (int i = 0; i < 2; ++i) copy16(reinterpret_cast<char*>(dst) + tok_at(lane, i), here > 8 * i ? p + 8 * i : src, here > 8 * i ? 16 : 0);
            } else {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t y = 2 * i < here ? reinterpret_cast<const uint16_t*>(p)[2 * i] : 0u;
                    const uint32_t z = 2 * i + 1 < here ? reinterpret_cast<const uint16_t*>(p)[2 * i + 1] : 0u;
                    w[i] = y | z << 16;
                }
                *reinterpret_cast<uint4*>(reinterpret_cast<char*>(dst) + tok_at(lane, 0)) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(reinterpret_cast<char*>(dst) + tok_at(lane, 1)) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (i & 1), r = g + (i < 2 ? 0 : 8);
                    const bool ok = t < s.L && r < rows;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(sm100::smem_u32(&dst[j * 32 + lane]) + 4 * i), "l"(ok ? src + (size_t)t * s.dv + r : src), "r"(ok ? 4 : 0) : "memory");
                }
        }
    };
    auto frag_tok = [&](const float4* src, float (&x)[4][4]) {  // in accumulator order: rows g, g + 8, pairs of tokens
        if (KT == 1) {
            uint32_t w[2][4];
            ldsm4_t(w[0], addr_tok(sm100::smem_u32(src), 0, lane));
            ldsm4_t(w[1], addr_tok(sm100::smem_u32(src), 1, lane));
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t z = w[j >> 1][(j & 1) * 2 + y];
                    x[j][2 * y] = __uint_as_float(z << 16);
                    x[j][2 * y + 1] = __uint_as_float(z & 0xffff0000u);
                }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 y = src[j * 32 + lane];
                x[j][0] = y.x; x[j][1] = y.y; x[j][2] = y.z; x[j][3] = y.w;
            }
        }
    };
    auto load_ahead = [&](int i) {  // dO and S Q^T of step i
        if (i >= nch || !active) return;
        const int c = nch - 1 - i;
        X& x = xb[i & 1];
        load_tok(x.d_o[0], d_o, c);
        const float4* src = reinterpret_cast<const float4*>(a.ws + a.l.sq) + (((size_t)n * nch + c) * a.l.slices + slice) * 128;
#pragma unroll
        for (int j = 0; j < 4; ++j) copy16(&x.sq[j][lane], src + j * 32 + lane, 16);
    };
    auto load_behind = [&](int i) {  // e and S K^T of step i
        if (i >= nch || !active) return;
        const int c = nch - 1 - i;
        X& x = xb[i & 1];
        const size_t at = (((size_t)n * nch + c) * a.l.slices + slice) * 128;
        const uint4* src = reinterpret_cast<const uint4*>(a.ws + a.l.e) + at;
        const float4* sk = reinterpret_cast<const float4*>(a.ws + a.l.sk) + at;
#pragma unroll
        for (int j = 0; j < 4; ++j) copy16(&x.sk[j][lane], sk + j * 32 + lane, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) copy16(&x.e[j >> 1][j & 1][lane], src + j * 32 + lane, 16);
    };
    // Of the last two chunks prepared: eta of the lane's tokens; of token `tok`, scale b dO . S q and the factors of dP . S k and of e . X k
    const int tok = (g >> 1) * 8 + 2 * c4 + (g & 1);  // sum_rows leaves a lane this token's sum
    float et[2][4][2], by_q[2] = {0.0f, 0.0f}, by_k[2] = {0.0f, 0.0f}, by_x[2] = {0.0f, 0.0f}, x_inv = 1.0f;
    auto prepare = [&](int i, int st) {
        X& x = xb[i & 1];
        const uint32_t as = ring + st * SB + AT_A;
        const float* sc = reinterpret_cast<const float*>(smem + st * SB + AT_SC);
        const float* head = sc + kRecHead * 32;
        float d[4][4], sums[8], m = 0.0f;
        frag_tok(x.d_o[0], d);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 y = x.sq[j][lane];
            sums[2 * j] = fmaf(d[j][0], y.x, d[j][2] * y.z);
            sums[2 * j + 1] = fmaf(d[j][1], y.y, d[j][3] * y.w);
            m = fmaxf(m, fmaxf(fmaxf(fabsf(d[j][0]), fabsf(d[j][1])), fmaxf(fabsf(d[j][2]), fabsf(d[j][3]))));
        }
        m = warp_most(m);
        const size_t at = ((size_t)n * nch + nch - 1 - i) * a.l.slices + slice;
        const float c_inv = reinterpret_cast<const float*>(a.ws + a.l.c_inv)[at];
        if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.max_do)[at] = m;
        by_q[0] = by_q[1]; by_k[0] = by_k[1]; by_x[0] = by_x[1];
        by_q[1] = sum_rows(sums, lane) * sc[kRecBq * 32 + tok] * c_inv;
        by_k[1] = sc[kRecBk * 32 + tok] * c_inv;
        by_x[1] = sc[kRecW * 32 + tok];
        float f, q;
        pow2_scale(m, f, q);
        float in[4][4] = {}, il[4][4] = {};
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            uint32_t hi[4], lo[4];
            to_a(d[2 * kk], d[2 * kk + 1], f, f, hi, lo);  // with bf16 one term, exactly
#pragma unroll
            for (int h = 0; h <= kk; ++h) {
                uint32_t bh[4], bl[4];
                ldsm4_t(bh, addr_kn<32>(as, 2 * h, kk, lane));
                ldsm4_t(bl, addr_kn<32>(as + 2048, 2 * h, kk, lane));
                mma(in[2 * h], hi, bh[0], bh[1]); mma(in[2 * h + 1], hi, bh[2], bh[3]);
                mma(il[2 * h], hi, bl[0], bl[1]); mma(il[2 * h + 1], hi, bl[2], bl[3]);
                if (KT == 2) { mma(il[2 * h], lo, bh[0], bh[1]); mma(il[2 * h + 1], lo, bh[2], bh[3]); }
            }
        }
        q *= head[kHeadAr];
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 y = make_float4((in[j][0] + il[j][0]) * q, (in[j][1] + il[j][1]) * q, (in[j][2] + il[j][2]) * q, (in[j][3] + il[j][3]) * q);
            x.in[j][lane] = y;
            most = fmaxf(most, fmaxf(fmaxf(fabsf(y.x), fabsf(y.y)), fmaxf(fabsf(y.z), fabsf(y.w))));
        }
        most = warp_most(most);
        const float qm = m * warp_most(fabsf(sc[kRecBq * 32 + lane]));
        float fq, q_inv;
        pow2_bound(qm, fq, q_inv);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 bq = *reinterpret_cast<const float2*>(sc + kRecBq * 32 + j * 8 + 2 * c4);
            const float2 e2 = *reinterpret_cast<const float2*>(sc + kRecEta * 32 + j * 8 + 2 * c4);
            et[0][j][0] = et[1][j][0]; et[0][j][1] = et[1][j][1];
            et[1][j][0] = e2.x; et[1][j][1] = e2.y;
            d[j][0] = d[j][0] * bq.x * fq; d[j][1] = d[j][1] * bq.y * fq; d[j][2] = d[j][2] * bq.x * fq; d[j][3] = d[j][3] * bq.y * fq;
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            uint32_t hi[4], lo[4];
            split_a(d[2 * kk], d[2 * kk + 1], hi, lo);
            x.q[0][kk][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            x.q[1][kk][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        if (lane == 0) { x.in_max = most; x.q_max = qm; x.q_inv = q_inv; x.q_sum = m * head[kHeadQsum]; }
    };
    // step i's dV, sums and fragments; `older`: one more chunk has been prepared since
    auto finish = [&](int i, bool older) {
        const int c = nch - 1 - i;
        X& x = xb[i & 1];
        const size_t at_max = ((size_t)n * nch + c) * a.l.slices + slice;
        const int own = older ? 0 : 1;
        float z[4][4], xk[4][4], part_[8], part_x[8], m = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 y = x.z[j][lane], w = KS == 1 ? x.in[j][lane] : x.xk[KS > 1 ? j : 0][KS > 1 ? lane : 0];
            z[j][0] = y.x; z[j][1] = y.y; z[j][2] = y.z; z[j][3] = y.w;
            xk[j][0] = w.x; xk[j][1] = w.y; xk[j][2] = w.z; xk[j][3] = w.w;
        }
        const float e_inv = reinterpret_cast<const float*>(a.ws + a.l.e_inv)[at_max];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint4 u = x.e[0][kk][lane], w = x.e[1][kk][lane];
            const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, ww[4] = {w.x, w.y, w.z, w.w};
            float e[4][2];
#pragma unroll
            for (int r = 0; r < 4; ++r) join_terms(uw[r], ww[r], e[r][0], e[r][1]);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float (&zz)[4] = z[2 * kk + j], (&xx)[4] = xk[2 * kk + j];
                    part_[4 * kk + 2 * j + y] = fmaf(zz[y], e[2 * j][y], zz[2 + y] * e[2 * j + 1][y]);
                    part_x[4 * kk + 2 * j + y] = fmaf(xx[y], e[2 * j][y], xx[2 + y] * e[2 * j + 1][y]);
                }
        }
        const size_t at = at_max * kDeltaChunk + tok;
        reinterpret_cast<float*>(a.ws + a.l.part_eta)[at] = sum_rows(part_, lane) * e_inv;
        reinterpret_cast<float*>(a.ws + a.l.part_x)[at] = sum_rows(part_x, lane) * e_inv * (by_x[own] * x_inv);
        const float (&eta)[4][2] = et[own];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 y = x.sk[j][lane];
            z[j][0] *= eta[j][0]; z[j][1] *= eta[j][1]; z[j][2] *= eta[j][0]; z[j][3] *= eta[j][1];  // dP = dV
            part_[2 * j] = fmaf(y.x, z[j][0], y.z * z[j][2]);
            part_[2 * j + 1] = fmaf(y.y, z[j][1], y.w * z[j][3]);
            m = fmaxf(m, fmaxf(fmaxf(fabsf(z[j][0]), fabsf(z[j][1])), fmaxf(fabsf(z[j][2]), fabsf(z[j][3]))));
        }
        reinterpret_cast<float*>(a.ws + a.l.part_s)[at] = fmaf(-sum_rows(part_, lane), by_k[own], by_q[own]);
        float sp, ip;
        pow2_scale(warp_most(m), sp, ip);
        uint4* dst = reinterpret_cast<uint4*>(a.ws + a.l.dp) + at_max * 64 * KT;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            uint32_t hi[4], lo[4];
            to_a(z[2 * kk], z[2 * kk + 1], sp, sp, hi, lo);
            dst[kk * 32 + lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            uint4* second = KT == 2 ? dst + 64 : reinterpret_cast<uint4*>(a.ws + a.l.dp_lo) + at_max * 64;
            second[kk * 32 + lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.dp_inv)[at_max] = ip;
        if (KT == 1) {
            const uint32_t tile = sm100::smem_u32(x.out);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                stsm4_t(addr_tok(tile, h, lane), pack_bf16(z[2 * h][0], z[2 * h][1]), pack_bf16(z[2 * h][2], z[2 * h][3]),
                        pack_bf16(z[2 * h + 1][0], z[2 * h + 1][1]), pack_bf16(z[2 * h + 1][2], z[2 * h + 1][3]));
            __syncwarp();
            const int t = c * kDeltaChunk + lane;
            const char* row = reinterpret_cast<const char*>(x.out);
            const uint4 y0 = *reinterpret_cast<const uint4*>(row + tok_at(lane, 0)), y1 = *reinterpret_cast<const uint4*>(row + tok_at(lane, 1));
            if (t < s.L) {
                IO* p = dv + (size_t)t * s.dv;
                if (vec) {
                    reinterpret_cast<uint4*>(p)[0] = y0;
                    if (rows > 8) reinterpret_cast<uint4*>(p)[1] = y1;
                } else {
                    const uint32_t w[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (2 * k < rows) reinterpret_cast<uint16_t*>(p)[2 * k] = (uint16_t)w[k];
                        if (2 * k + 1 < rows) reinterpret_cast<uint16_t*>(p)[2 * k + 1] = (uint16_t)(w[k] >> 16);
                    }
                }
            }
            __syncwarp();
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (y & 1), r = g + (y < 2 ? 0 : 8);
                    if (t < s.L && r < rows) dv[(size_t)t * s.dv + r] = from_f32<IO>(z[j][y]);
                }
        }
    };
    auto save_x = [&](int i) {  // X behind step i's chunk, where a block ends there
        const int c = nch - 1 - i;
        if (lane != 0 || !((c & 1) || c == nch - 1)) return;
        const X& x = xb[i & 1];
        const size_t at = ((size_t)n * a.l.nblk + (c >> 1)) * a.l.slices + slice;
        bulk_store(a.ws + a.l.X + at * a.l.state_bytes * KT, sm100::smem_u32(x.x), (uint32_t)a.l.state_bytes * KT);
        reinterpret_cast<float*>(a.ws + a.l.x_inv)[at] = x.x_inv;
    };
    auto near_s = [&](int i) {  // the state that the chain takes its inner product with in step i, into L2
        const int c = nch - 1 - i;
        if (i >= nch || !active || (c & 1) || lane * 128 >= (int)a.l.state_bytes) return;
        const size_t at = ((size_t)n * a.l.nblk + (c >> 1)) * a.l.slices + slice;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(a.ws + a.l.S + at * a.l.state_bytes + lane * 128));
        asm volatile("prefetch.global.L2 [%0];" ::"l"(a.ws + a.l.S_lo + at * a.l.state_bytes + lane * 128));
    };
    load_ahead(0);
    asm volatile("cp.async.commit_group;" ::: "memory");
    load_ahead(1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
    wait_phase(&full[0], 0, wait, 904);
    if (active) prepare(0, 0);
    __syncthreads();
    int st = 0, phase_next = 0;
    for (int i = 0; i < nch; ++i) {
        const int st_next = st + 1 == NS ? 0 : st + 1;
        if (st_next == 0) phase_next ^= 1;
        load_ahead(i + 2);
        load_behind(i);
        near_s(i + 2);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        const float x_inv_next = xb[i & 1].x_inv;  // the chain gives that place another value while finish(i) runs
        if (active) save_x(i);
        bulk_store_commit();
        if (active && i > 0) finish(i - 1, true);
        x_inv = x_inv_next;
        if (i + 1 < nch) {
            wait_phase(&full[st_next], phase_next, wait, 904);
            if (active) prepare(i + 1, st_next);
        }
        bulk_store_read();  // the chain may write X there again
        __syncthreads();
        if (fetches && i + NS < nch) fetch(i + NS, st);
        __syncwarp();
        st = st_next;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    if (active) finish(nch - 1, false);
    bulk_store_done();
}

// d eta and d log_gamma: a warp per chunk, the two chunks of a block beside each other.  dO_s . e_i and dP_s . e_i over all value rows are products of the
// fragments that the walks left (rows to columns by transposing 8 x 8 matrices in registers), both terms of every operand; A and D K K^T come from
// the chunk's record.  The sums over i < t <= s are formed as they stand, first over i, then over s.  B = b_end <X, S_0> comes from the walk for a
// block's first chunk, whose S_0 is kept.  For the second one it is what reaches this chunk at all, which is its first token's gradient and known from the
// first chunk (B and all X terms there), without what its tokens read (all S terms).  That difference is the one place where terms cancel, down to
// another token's gradient in 32 bits; where the chunk forgets everything, B is 0.
// Bound by fetching the fragments: 64 heads of 4096 tokens, 128 x 128, bf16, in 100 us (390 MB: 3.9 TB/s); 96 of 2048, 64 x 64, in 50 us.
template <typename IO, int KT>
__global__ void __launch_bounds__(kGateWarps * 32) delta_gate_kernel(const DeltaBwdArgs ba, const bool pairs) {
    __shared__ float grid[kGateWarps][32][33];
    __shared__ double handed[kGateWarps / 2];
    const DeltaArgs& a = ba.f;
    const DeltaShape& s = a.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const int64_t item = (int64_t)blockIdx.x * (kGateWarps / 2) + (warp >> 1), n = item / a.l.nblk;
    const int blk = (int)(item % a.l.nblk), c = 2 * blk + (warp & 1), t0 = c * kDeltaChunk;
    const bool here = item < a.l.N * a.l.nblk && c < a.l.nch;
    const float4* hx = reinterpret_cast<const float4*>(a.ws + a.l.hx) + (size_t)item * a.l.slices;
    double flow = 0.0, back = 0.0, forth = 0.0, through = 0.0;  // of token t = lane: what is handed on; S terms; X terms; B
    float de = 0.0f;
    bool forgets = false;
    if (here) {
        const char* rec = a.ws + a.l.rec + ((size_t)n * a.l.nch + c) * a.l.rec_bytes;
        float wo[6][4], wp[6][4];  // dO_s . e_i and dP_s . e_i
#pragma unroll
        for (int i = 0; i < 6; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) wo[i][x] = wp[i][x] = 0.0f;
        const IO* d_o = reinterpret_cast<const IO*>(ba.d_o) + ((size_t)n * s.L + t0) * s.dv;
        for (int sl = 0; sl < a.l.slices; ++sl) {
            const size_t at = ((size_t)n * a.l.nch + c) * a.l.slices + sl;
            const uint4* e4 = reinterpret_cast<const uint4*>(a.ws + a.l.e) + at * 128 + lane;
            const uint4* p4 = reinterpret_cast<const uint4*>(a.ws + a.l.dp) + at * 64 * KT + lane;
            const uint4* q4 = KT == 2 ? p4 + 64 : reinterpret_cast<const uint4*>(a.ws + a.l.dp_lo) + at * 64 + lane;
            const uint4 raw_e[2][2] = {{e4[0], e4[32]}, {e4[64], e4[96]}}, raw_p[2][2] = {{p4[0], p4[32]}, {q4[0], q4[32]}};
            const float e_inv = reinterpret_cast<const float*>(a.ws + a.l.e_inv)[at], p_inv = reinterpret_cast<const float*>(a.ws + a.l.dp_inv)[at];
            de += reinterpret_cast<const float*>(a.ws + a.l.part_eta)[at * kDeltaChunk + lane];
            back += reinterpret_cast<const float*>(a.ws + a.l.part_s)[at * kDeltaChunk + lane];
            forth += reinterpret_cast<const float*>(a.ws + a.l.part_x)[at * kDeltaChunk + lane];
            if (!(c & 1)) through += (hx[sl].x + hx[sl].y) + (hx[sl].z + hx[sl].w);
            float so, o_inv;
            pow2_scale(reinterpret_cast<const float*>(a.ws + a.l.max_do)[at], so, o_inv);
            // A operands: tokens x value rows of the slice.  [term][tokens 0-15, 16-31]
            uint32_t ao[KT][2][4], ap[2][2][4], b[2][4][2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = m * 16 + (r & 1) * 8 + g, d = sl * 16 + (r >> 1) * 8 + 2 * c4;
                    const IO* p = d_o + (size_t)t * s.dv + d;
                    const bool ok = t0 + t < s.L;
                    float y0 = 0.0f, y1 = 0.0f;
                    if (sizeof(IO) == 2 && pairs) {
                        if (ok && d < s.dv) {
                            const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
                            y0 = __uint_as_float(w << 16);
                            y1 = __uint_as_float(w & 0xffff0000u);
                        }
                    } else {
                        if (ok && d < s.dv) y0 = to_f32(p[0]);
                        if (ok && d + 1 < s.dv) y1 = to_f32(p[1]);
                    }
                    uint32_t hi, lo;
                    split(y0 * so, y1 * so, hi, lo);  // with bf16 one term, exactly
                    ao[0][m][r] = hi;
                    if (KT == 2) ao[KT - 1][m][r] = lo;
                }
            // fragments [value rows][tokens]: register r of k-step kk holds rows 8 (r & 1) .., tokens 16 kk + 8 (r >> 1) ..
#pragma unroll
            for (int term = 0; term < 2; ++term)
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const uint4 x = raw_e[term][kk], y = raw_p[term][kk];
                    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        b[term][2 * kk + (r >> 1)][r & 1] = transposed(xw[r]);
                        ap[term][kk][(r >> 1) + 2 * (r & 1)] = transposed(yw[r]);
                    }
                }
            const float fo = o_inv * e_inv, fp = p_inv * e_inv;
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                const int m = i < 2 ? 0 : 1, j = i < 2 ? i : i - 2;
                float y[4];
                mma0(y, ao[0][m], b[1][j][0], b[1][j][1]);
                if (KT == 2) mma(y, ao[KT - 1][m], b[0][j][0], b[0][j][1]);
                mma(y, ao[0][m], b[0][j][0], b[0][j][1]);
#pragma unroll
                for (int x = 0; x < 4; ++x) wo[i][x] = fmaf(y[x], fo, wo[i][x]);
                mma0(y, ap[0][m], b[1][j][0], b[1][j][1]);
                mma(y, ap[1][m], b[0][j][0], b[0][j][1]);
                mma(y, ap[0][m], b[0][j][0], b[0][j][1]);
#pragma unroll
                for (int x = 0; x < 4; ++x) wp[i][x] = fmaf(y[x], fp, wp[i][x]);
            }
        }
        const float4* pair = reinterpret_cast<const float4*>(rec + kDeltaRecPairs) + lane;
        const float* sc = reinterpret_cast<const float*>(rec + kDeltaRecSkip);
        float (&m)[32][33] = grid[warp];
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            const int m0 = i < 2 ? 0 : 16, n0 = i < 2 ? i * 8 : (i - 2) * 8;
            const float4 q = pair[i * 32], k = pair[(6 + i) * 32];
            const float qw[4] = {q.x, q.y, q.z, q.w}, kw[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int t = m0 + g + (x >> 1) * 8, u = n0 + 2 * c4 + (x & 1);
                m[t][u] = u < t ? (qw[x] * wo[i][x] - kw[x] * wp[i][x]) * sc[kRecEta * 32 + u] : 0.0f;
            }
        }
        __syncwarp();
        float run = 0.0f;  // lane = s: sum over i < t for every t up to s
#pragma unroll 4
        for (int t = 0; t < 32; ++t) {
            const float x = t < lane ? m[lane][t] : 0.0f;
            m[lane][t] = t <= lane ? run : 0.0f;
            run += x;
        }
        __syncwarp();
#pragma unroll 4
        for (int t = 0; t < 32; ++t) flow += m[t][lane];  // lane = t: over s >= t
        // S terms from t on, X terms before t, and all of either
        double after = back, before = __shfl_up_sync(kAll, forth, 1);
        if (lane == 0) before = 0.0;
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            const double y = __shfl_down_sync(kAll, after, i), z = __shfl_up_sync(kAll, before, i);
            if (lane + i < 32) after += y;
            if (lane >= i) before += z;
        }
        flow += after + before;
        back = __shfl_sync(kAll, after, 0);
        forth = __shfl_sync(kAll, before + forth, 31);
        const float end = sc[kRecHead * 32 + kHeadEnd];
        forgets = end == 0.0f;
        if (!(c & 1)) {
            through *= end;
            if (lane == 0) handed[warp >> 1] = through + forth;
        }
    }
    __syncthreads();
    if (!here) return;
    if ((c & 1) && !forgets) through = handed[warp >> 1] - back;
    flow += through;
    const int t = t0 + lane;
    if (t >= s.L) return;
    const size_t out = (size_t)n * s.L + t;
    ba.d_eta[out] = de;
    ba.d_log_gamma[out] = a.log_gamma[out] < -104.0f ? 0.0f : (float)flow;  // a decay that is 0 in 32 bits has none
}

// ---- dQ and dK ----------------------------------------------------------------------------------------------------
// A CTA takes 64 tokens of one query / key head and adds up the value heads of its group.  Sixteen warps: 16 tokens times a quarter of the key
// columns each.  The value rows come through shared memory ROWS at a time, with S_0 (dQ's and dK's first part, both token-by-token matrices) and
// again with X; what the chains left in fragment order goes into tiles of rows here, at one scale for all slices (S, X) or all of a chunk (e, dP, dO).  With bf16 I/O one term of every
// operand serves: dQ and dK are off by 2^-11 of their terms before they are rounded to 2^-8.  AHEAD: the next head's raw tiles come by bulk copies.
// Bound by the dependent phases of a head (tiles, products with S, token matrices, products with X, products with K and Q, a barrier between any
// two): 20 thousand cycles, of which the MMAs are 5, the tiles 4.  4 x 4 key heads of 4 value heads, 4096 tokens, 128 x 128, bf16: 348 us (470 MB: 1.35
// TB/s); 8 x 12 heads, 2048 tokens, 64 x 64: 209 us.
// One term leaves dq and dk 1.68e-3 from their values in 64 bits where rounding alone leaves 1.66e-3.  Both terms of S, e, dP, X and the token matrices are 2.5 times
// the MMAs and twice the tiles, without room for the next head's: 778 and 301 us.  A caller who wants them has fp32 I/O.
template <int DK, int KT> constexpr int qk_rows() { return KT == 1 ? DK : 32; }
template <int DK, int KT> constexpr int qk_ctas() { return KT == 1 && DK == 64 ? 2 : 1; }  // per SM
template <int DK, int KT> constexpr int qk_work() {
    return 2 * KT * 128 * DK + KT * qk_rows<DK, KT>() * (2 * DK + 3 * 128) + 2 * KT * 8192 + 2 * 64 * 8 + 2 * 3 * 256 + 640;
}
// with bf16, what the next head's tiles are made of: a state (S, then X) and the first terms of e and dP of two chunks as the chains left them, dO's rows
template <int DK, int KT, bool AHEAD> constexpr int qk_smem() {
    constexpr int SL = qk_rows<DK, KT>() / 16;
    return qk_work<DK, KT>() + (AHEAD ? SL * (32 * DK + 3 * 2048) : 0);
}

template <typename IO, int DK, int KT, bool AHEAD>
__global__ void __launch_bounds__(512, qk_ctas<DK, KT>()) delta_qk_kernel(const DeltaBwdArgs ba, const bool vec) {
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
    double* run2 = reinterpret_cast<double*>(mat + 2 * KT * 8192);  // [2][64], of this head and of the next
    float* bt2 = reinterpret_cast<float*>(run2 + 2 * 64);          // [2][3][64]: b, eta D_end, eta
    float* scl2 = bt2 + 2 * 3 * 64;                                // [2][64]: the scales and the slices' ratios to them
    float* red = scl2 + 2 * 64;                                    // 32
    const uint32_t ks = sm100::smem_u32(kq), qs = ks + KT * 128 * DK, ss = sm100::smem_u32(st_s), os = sm100::smem_u32(st_o),
                   us = sm100::smem_u32(st_u), ps = sm100::smem_u32(st_p), ms = sm100::smem_u32(mat);
    const int nchunks = min(2, a.l.nch - 2 * blk);
    // The raw tiles of a head come by bulk copies while the head before is worked on: S behind X's use, e, dP and dO behind their own
    char* raw_s = smem + qk_work<DK, KT>();
    char* raw_e = raw_s + SL * 32 * DK;  // [chunk][slice] of 1 KB
    char* raw_p = raw_e + SL * 2048;
    char* raw_o = raw_p + SL * 2048;  // [64 tokens][dv]
    __shared__ uint64_t come[3];  // S, X, e with dP and dO
    __shared__ int dead_flag;
    sm100::WaitCtx wait{&dead_flag, reinterpret_cast<int*>(a.ws)};
    const int64_t n_first = (nk / s.Hk) * s.H + (nk % s.Hk) * r;
    // by one warp, a copy a lane
    auto fetch_state = [&](int64_t n, size_t off, uint64_t* bar) {
        if (lane != 0) return;
        const uint32_t bytes = (uint32_t)(a.l.slices * a.l.state_bytes);
        sm100::mbar_expect_tx(bar, bytes);
        bulk_copy(sm100::smem_u32(raw_s), a.ws + off + ((size_t)n * a.l.nblk + blk) * a.l.slices * a.l.state_bytes, bytes, bar);
    };
    auto fetch_tok = [&](int64_t n) {
        const uint32_t rows = vec ? (uint32_t)(min(kDeltaBlock, s.L - t0) * s.dv * 2) : 0;
        if (lane == 0) sm100::mbar_expect_tx(&come[2], (uint32_t)(nchunks * a.l.slices * 2048) + rows);
        __syncwarp();
        const int ch = (lane >> 3) & 1, sl = lane & 7;
        const size_t at = ((size_t)n * a.l.nch + 2 * blk + ch) * a.l.slices;
        if (lane < 16 && ch < nchunks && sl < a.l.slices)
            bulk_copy(sm100::smem_u32(raw_e + (ch * SL + sl) * 1024), a.ws + a.l.e + (at + sl) * 2048, 1024, &come[2]);
        if (lane >= 16 && sl == 0 && ch < nchunks)
            bulk_copy(sm100::smem_u32(raw_p + ch * SL * 1024), a.ws + a.l.dp + at * 1024, (uint32_t)(a.l.slices * 1024), &come[2]);
        if (lane == 31 && rows) bulk_copy(sm100::smem_u32(raw_o), reinterpret_cast<const IO*>(ba.d_o) + ((size_t)n * s.L + t0) * s.dv, rows, &come[2]);
    };
    const bool fetches = AHEAD && warp == 1;
    if (fetches) {
        if (lane == 0) {
            for (int i = 0; i < 3; ++i) sm100::mbar_init(&come[i], 1);
            dead_flag = 0;
            sm100::fence_mbar_init();
        }
        __syncwarp();
        fetch_state(n_first, a.l.S, &come[0]);
        fetch_tok(n_first);
    }
    // the two chunks' tiles at one scale
    float ik, iq;
    {
        const float* h0 = reinterpret_cast<const float*>(a.ws + a.l.rec + ((size_t)n_first * a.l.nch + 2 * blk) * a.l.rec_bytes + 8192) + kRecHead * 32;
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
                if (y != 1.0f) x = times_ratio(x, y);
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
    // Decays, learning rates and scales of a head, by two warps with few products (16-token rows that see only themselves); with AHEAD, loaded before
    // the products of the head before and made from that behind them.
    const bool decays = warp == 2, scales = warp == 3;
    auto setup_load = [&](int64_t n, float (&x)[5]) {
        if (decays) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int t = t0 + 2 * lane + k;
                x[k] = t < s.L ? a.log_gamma[(size_t)n * s.L + t] : 0.0f;
                x[2 + k] = t < s.L ? a.eta[(size_t)n * s.L + t] : 0.0f;
            }
        } else {  // lane = slice and chunk
            const int sl = lane & 7, ch = lane >> 3;
            const bool ok = sl < a.l.slices, tok = ok && ch < nchunks;
            const size_t at = ((size_t)n * a.l.nch + 2 * blk + ch) * a.l.slices + sl, at_s = ((size_t)n * a.l.nblk + blk) * a.l.slices + sl;
            x[0] = tok ? reinterpret_cast<const float*>(a.ws + a.l.e_inv)[at] : 0.0f;
            x[1] = tok ? reinterpret_cast<const float*>(a.ws + a.l.dp_inv)[at] : 0.0f;
            x[2] = tok ? reinterpret_cast<const float*>(a.ws + a.l.max_do)[at] : 0.0f;
            x[3] = ok ? reinterpret_cast<const float*>(a.ws + a.l.s_inv)[at_s] : 0.0f;
            x[4] = ok ? reinterpret_cast<const float*>(a.ws + a.l.x_inv)[at_s] : 0.0f;
        }
    };
    auto setup_make = [&](const float (&x)[5], int buf) {
        if (decays) {
            double* run = run2 + buf * 64;
            float* bt = bt2 + buf * 192;
            const double g0 = x[0] < -1000.0f ? -1000.0f : x[0], sum = g0 + (double)(x[1] < -1000.0f ? -1000.0f : x[1]);
            double acc = sum;
#pragma unroll
            for (int i = 1; i < 32; i <<= 1) {
                const double y = __shfl_up_sync(kAll, acc, i);
                if (lane >= i) acc += y;
            }
            const double end = __shfl_sync(kAll, acc, 31), before = acc - sum;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const double y = before + (k ? sum : g0);
                run[2 * lane + k] = y;
                bt[2 * lane + k] = expf((float)y);
                bt[64 + 2 * lane + k] = expf((float)(end - y)) * x[2 + k];
                bt[128 + 2 * lane + k] = x[2 + k];
            }
        } else {
            float* scl = scl2 + buf * 64;
            // e, dP and dO: a scale per chunk, as no product sums over tokens of theirs; S and X have one
            float iu = x[0], ip = x[1], mo = x[2];
#pragma unroll
            for (int i = 1; i < 8; i <<= 1) {
                iu = fmaxf(iu, __shfl_xor_sync(kAll, iu, i));
                ip = fmaxf(ip, __shfl_xor_sync(kAll, ip, i));
                mo = fmaxf(mo, __shfl_xor_sync(kAll, mo, i));
            }
            if (iu == 0.0f) iu = ip = 1.0f;  // no second chunk
            const float iS = warp_most(x[3]), iX = warp_most(x[4]);
            float so, io;
            pow2_scale(mo, so, io);
            if (lane < 16 && (lane & 7) == 0) {
                float* of = scl + (lane >> 3);
                of[0] = iu; of[2] = ip; of[4] = so; of[6] = io;
            }
            if (lane == 0) { scl[8] = iS; scl[9] = iX; }
            // what brings a slice's fragments to these scales: powers of two, at most 1
            if (lane < 16) {
                scl[16 + lane] = x[0] / iu;
                scl[32 + lane] = x[1] / ip;
            }
            if (lane < 8) {
                scl[48 + lane] = x[3] / iS;
                scl[56 + lane] = x[4] / iX;
            }
        }
    };
    float next[5] = {};
    if (AHEAD && (decays || scales)) {
        setup_load(n_first, next);
        setup_make(next, 0);
    }
    for (int hd = 0; hd < r; ++hd) {
        const int64_t n = n_first + hd;
        const int buf = AHEAD ? hd & 1 : 0;
        const double* run = run2 + buf * 64;
        const float *bt = bt2 + buf * 192, *dend = bt + 64, *eta = bt + 128, *scl = scl2 + buf * 64;
        // fragments [16 value rows][16 columns] of a slice to rows of a tile
        auto put = [&](char* tile, int cols, int row, int piece, const uint4& x, float ratio) {
            const uint4 y = times_ratio(x, ratio);
            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = row + (i & 1) * 8, pp = piece + (i >> 1);
                const uint32_t at = cols == 64 ? tile_at<64>(rr, pp) : tile_at<DK>(rr, pp);
                *reinterpret_cast<uint32_t*>(tile + at + c4 * 4) = w[i];
            }
        };
        // a tile's fragments, all loads under way before the first is looked at, and what then becomes of them; a warp per (term, slice, ..)
        constexpr int QT = SL * 4 * KT * 32 / 512, QS = SL * KT * (DK / 16) / 16;
        auto load_tok = [&](size_t off, int terms, const char* raw, uint4 (&x)[QT], int sl0) {
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                const int i = warp + 16 * q, kk = i & 1, ch = (i >> 1) & 1, sl = (i >> 2) % SL, term = (i >> 2) / SL;
                x[q] = make_uint4(0, 0, 0, 0);
                if (sl0 + sl >= a.l.slices || ch >= nchunks) continue;
                const size_t at = ((size_t)n * a.l.nch + 2 * blk + ch) * a.l.slices + sl0 + sl;
                x[q] = AHEAD ? reinterpret_cast<const uint4*>(raw)[(ch * SL + sl) * 64 + kk * 32 + lane]
                             : reinterpret_cast<const uint4*>(a.ws + off)[(at * terms + term) * 64 + kk * 32 + lane];
            }
        };
        auto put_tok = [&](const float* ratios, char* dst, const uint4 (&x)[QT], int sl0) {
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                const int i = warp + 16 * q, kk = i & 1, ch = (i >> 1) & 1, sl = (i >> 2) % SL, term = (i >> 2) / SL;
                put(dst + term * TT, 64, sl * 16 + g, (ch * 2 + kk) * 2, x[q], ratios[ch * 8 + ((sl0 + sl) & 7)]);
            }
        };
        auto load_state = [&](size_t off, size_t off_lo, int terms, uint4 (&x)[QS], int sl0) {
#pragma unroll
            for (int q = 0; q < QS; ++q) {
                const int i = warp + 16 * q, kk = i % (DK / 16), sl = i / (DK / 16) % SL, term = i / (DK / 16) / SL;
                x[q] = make_uint4(0, 0, 0, 0);
                if (sl0 + sl >= a.l.slices) continue;
                const size_t at = ((size_t)n * a.l.nblk + blk) * a.l.slices + sl0 + sl;
                const char* src = off_lo ? a.ws + (term ? off_lo : off) + at * a.l.state_bytes : a.ws + off + (at * terms + term) * a.l.state_bytes;
                x[q] = reinterpret_cast<const uint4*>(AHEAD ? raw_s + sl * 32 * DK : src)[kk * 32 + lane];
            }
        };
        auto put_state = [&](const float* ratios, const uint4 (&x)[QS], int sl0) {
#pragma unroll
            for (int q = 0; q < QS; ++q) {
                const int i = warp + 16 * q, kk = i % (DK / 16), sl = i / (DK / 16) % SL, term = i / (DK / 16) / SL;
                put(st_s + term * TS, DK, sl * 16 + g, kk * 2, x[q], ratios[(sl0 + sl) & 7]);
            }
        };
        uint4 xs[QS], xe[QT], xp[QT];
        auto load_all = [&](int sl0) {
            load_state(a.l.S, KT == 2 ? a.l.S_lo : 0, 1, xs, sl0);
            load_tok(a.l.e, 2, raw_e, xe, sl0);
            load_tok(a.l.dp, KT, raw_p, xp, sl0);
        };
        if (!AHEAD) {
            __syncthreads();
            if (decays || scales) {
                float x[5];
                setup_load(n, x);
                setup_make(x, 0);
            }
        }
        __syncthreads();  // this head's scales are there, the one before has been read
        // of the chunk of the warp's rows (with e's of its columns for the token matrices)
        const float iu = scl[tw >> 1], ip = scl[2 + (tw >> 1)], io = scl[6 + (tw >> 1)], iu_col = scl[hw >> 1], iS = scl[8], iX = scl[9];
        auto stage_do = [&](int d0) {  // [64 tokens][ROWS value rows]
#pragma unroll
            for (int q = 0; q < 64 * ROWS / 8 / 512 + (64 * ROWS / 8 < 512); ++q) {
                const int i = tid + 512 * q, row = i / (ROWS / 8), piece = i % (ROWS / 8), t = t0 + row, d = d0 + piece * 8;
                if (row >= 64) continue;
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = 0.0f;
                if (t < s.L && d < s.dv) {
                    const IO* p = AHEAD && vec ? reinterpret_cast<const IO*>(raw_o) + row * s.dv + d
                                               : reinterpret_cast<const IO*>(ba.d_o) + ((size_t)n * s.L + t) * s.dv + d;
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
                const float so = scl[4 + (row >> 5)];
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
            if (AHEAD) {  // from shared memory, one after the other: nothing to wait for together
                wait_phase(&come[0], hd & 1, wait, 905);
                wait_phase(&come[2], hd & 1, wait, 906);
                load_state(a.l.S, 0, 1, xs, 0);
                put_state(scl + 48, xs, 0);
                load_tok(a.l.e, 2, raw_e, xe, 0);
                put_tok(scl + 16, st_u, xe, 0);
                load_tok(a.l.dp, KT, raw_p, xp, 0);
                put_tok(scl + 32, st_p, xp, 0);
                stage_do(0);
            } else {
                load_all(sl0);
                stage_do(sl0 * 16);
                put_state(scl + 48, xs, sl0);
                put_tok(scl + 16, st_u, xe, sl0);
                put_tok(scl + 32, st_p, xp, sl0);
                if (a.l.slices <= SL) load_state(a.l.X, 0, KT, xs, 0);  // for behind these products
            }
            __syncthreads();
            if (fetches) {  // everything has been read
                fetch_state(n, a.l.X, &come[1]);
                if (hd + 1 < r) fetch_tok(n + 1);
            }
            const bool another = AHEAD && (decays || scales) && hd + 1 < r;
            if (another) setup_load(n + 1, next);
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
            if (another) setup_make(next, (hd + 1) & 1);
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
                sg[j][x] = u <= t ? sg[j][x] * (io * iu_col) * (D * s.scale) : 0.0f;
                kp[j][x] = u < t ? -kp[j][x] * (ip * iu_col) * D : 0.0f;
                m0 = fmaxf(m0, fabsf(sg[j][x]));
                m1 = fmaxf(m1, fabsf(kp[j][x]));
            }
        m0 = warp_max(m0); m1 = warp_max(m1);
        if (lane == 0) { red[warp] = m0; red[16 + warp] = m1; }
        if (AHEAD) {
            wait_phase(&come[1], hd & 1, wait, 907);
            load_state(a.l.X, 0, KT, xs, 0);
        }
        if (a.l.slices <= SL) put_state(scl + 56, xs, 0);  // the products with S are through
        __syncthreads();
        if (fetches && hd + 1 < r) fetch_state(n + 1, a.l.S, &come[0]);
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
                load_tok(a.l.e, 2, raw_e, xe, sl0);
                load_state(a.l.X, 0, KT, xs, sl0);
                put_tok(scl + 16, st_u, xe, sl0);
                put_state(scl + 56, xs, sl0);
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

template <typename IO, int DK, int KT, int KS> int launch_chain(const DeltaBwdArgs& b, int per, bool vec, cudaStream_t st) {
    static_assert(chain_smem<DK, KT, KS>(KS > 1 ? 1 : KT == 1 ? 4 : 2) <= kMostSharedMemory, "shared memory of the chain");
    const int bytes = chain_smem<DK, KT, KS>(per);
    auto kernel = delta_chain_kernel<IO, DK, KT, KS>;
    const cudaError_t e = allow_shared_memory<delta_chain_kernel<IO, DK, KT, KS>>();
    if (e != cudaSuccess) return (int)e;
    kernel<<<(unsigned)(b.f.l.N * ((b.f.l.slices + per - 1) / per)), per * (KS + 1) * 32, bytes, st>>>(b, per, vec);
    return (int)cudaGetLastError();
}

template <typename IO, int DK, int KT, bool AHEAD> int launch_qk(const DeltaBwdArgs& b, cudaStream_t st) {
    constexpr int bytes = qk_smem<DK, KT, AHEAD>();
    static_assert(bytes * qk_ctas<DK, KT>() <= kMostSharedMemory, "shared memory of the dq / dk kernel");
    auto kernel = delta_qk_kernel<IO, DK, KT, AHEAD>;
    const cudaError_t e = allow_shared_memory<delta_qk_kernel<IO, DK, KT, AHEAD>>();
    if (e != cudaSuccess) return (int)e;
    const bool vec = b.f.s.dv % 8 == 0 && reinterpret_cast<uintptr_t>(b.d_o) % 16 == 0;
    kernel<<<(unsigned)(b.f.l.Nk * b.f.l.nblk), 512, bytes, st>>>(b, vec);
    return (int)cudaGetLastError();
}

template <typename IO, int DK, int KT> int launch(const DeltaBwdArgs& b, cudaStream_t st) {
    const DeltaArgs& a = b.f;
    {
        constexpr int most = KT == 1 ? 4 : 2;
        const bool vec = a.s.dv % 8 == 0 && (reinterpret_cast<uintptr_t>(b.d_o) | reinterpret_cast<uintptr_t>(b.dv)) % 16 == 0;
        // Few slices, as many as SMs at most: the columns of each over DK / 32 warps.  16 heads of 128 x 128, 4096 tokens, bf16, forward and reverse pass: 691 us, with a
        // warp per slice 727.  More: as the forward's.
        int rc;
        if (a.l.N * a.l.slices <= 148) {
            rc = launch_chain<IO, DK, KT, DK / 32>(b, 1, vec, st);
        } else {
            rc = launch_chain<IO, DK, KT, 1>(b, slices_per_cta(a.l, most), vec, st);
        }
        if (rc != 0) return rc;
    }
    // With bf16 the tiles of a head that fits (all but value rows beyond 64 with keys of up to 64) come ahead.  4 x 4 key heads with 4 value heads each, 4096
    // tokens, 128 x 128: 348 us, and 416 with loads when they are needed; 8 x 12 heads with one each, 2048 tokens, 64 x 64: 209 and 213.
    int rc;
    if constexpr (KT == 1 && DK == 128) rc = launch_qk<IO, DK, KT, true>(b, st);
    else if constexpr (KT == 1) rc = a.l.slices <= qk_rows<DK, KT>() / 16 ? launch_qk<IO, DK, KT, true>(b, st) : launch_qk<IO, DK, KT, false>(b, st);
    else rc = launch_qk<IO, DK, KT, false>(b, st);
    if (rc != 0) return rc;
    const bool pairs = a.s.dv % 2 == 0 && reinterpret_cast<uintptr_t>(b.d_o) % 4 == 0;
    constexpr int blocks = kGateWarps / 2;
    delta_gate_kernel<IO, KT><<<(unsigned)((a.l.N * a.l.nblk + blocks - 1) / blocks), kGateWarps * 32, 0, st>>>(b, pairs);
    return (int)cudaGetLastError();
}

}  // namespace

int delta_bwd_launch(const DeltaBwdArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.f.s.f32) return a.f.l.DK == 64 ? launch<float, 64, 2>(a, st) : launch<float, 128, 2>(a, st);
    return a.f.l.DK == 64 ? launch<__nv_bfloat16, 64, 1>(a, st) : launch<__nv_bfloat16, 128, 1>(a, st);
}

}  // namespace e2ttt
