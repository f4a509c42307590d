// Gated delta rule, the walk over the chunks.  A slice of 16 value rows of a sequence's state, [16, dk], stays in registers from the first
// token to the last (64 a lane of one warp at dk = 128, or shared out by columns over KS warps), and the slices of a sequence never meet but
// for the tiles that they share.
// Per chunk of 32 tokens, rows = value rows:  P = V - b S K^T,  e = P T^T,  O = b S Q^T + e (A eta)^T,  S = b_end S + (D_end u) K.
// Each product's result is the next one's A operand in place.  The chunk's tiles (queries, keys, T, A, scalars; written by
// delta_prep.cu) arrive by bulk copies, several chunks ahead.
// The chain P, e, S is what a chunk waits for; one more warp per slice does what hangs off it, a chunk behind: O from the state's and e's
// fragments (which the chain leaves in shared memory), and the values' loads and the outputs' stores.  One barrier a chunk.
// A chain is bound by the instructions of a chunk one after the other (an MMA every 8 cycles, 146 of them, and splitting the operands into
// terms), so scales are one per slice, folded into the scalars that the values are multiplied with anyway, and come from bounds that are known
// before the values are.
// 4 x 16 sequences of 4096 tokens, 128 x 128, bf16: 268 us (128 chunks, one after the other: 2.1 us each), 317 us with saved states (670 MB of states,
// errors and the states' products with queries and keys to write); 16 sequences of 32768 tokens: 1280 us (1024 chunks: 1.25 us each, one slice on an
// SM); 8 x 12 sequences of 2048 tokens, 64 x 64, with saved states: 121 us.
#include "api_checks.h"
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

template <int DK, int KT> constexpr int stage_bytes() { return 2 * KT * 64 * DK + kDeltaRecBytes; }
template <int KT> constexpr int stages() { return KT == 1 ? 4 : 3; }

// what the warps of a slice hand over, a buffer per parity of the chunk: fragments of S and e (both terms), what undoes their scales, the values of the next chunk (fp32 in fragment order, or bf16 tokens x rows) and a bound on them, the outputs on their way out
template <int DK, int KT, int KS> struct alignas(128) Exchange {
    uint4 s[2][DK / 16][32];
    uint4 u[2][2][32];
    float4 v[KT == 1 ? 2 : 4][32];
    uint4 o[KT == 1 ? 64 : 1];
    float4 part[KS > 1 ? KS : 1][4][KS > 1 ? 32 : 1];  // S K^T over a warp's columns (KS > 1)
    float norm[KS];                       // the sum of squares of its part of S, scaled
    float s_inv, u_inv, v_max;
};

template <int DK, int KT, int KS> constexpr int fwd_smem(int slices) {
    return stages<KT>() * stage_bytes<DK, KT>() + 2 * slices * (int)sizeof(Exchange<DK, KT, KS>);
}

// vec: bf16 rows of v and o that allow 16-byte pieces.
// SAVE: what the reverse pass reads is kept.
template <typename IO, int DK, int KT, int KS, bool SAVE>
__global__ void __launch_bounds__(KS == 1 ? 256 : 160, 1) delta_fwd_kernel(const DeltaArgs a, const int per, const bool vec) {
    extern __shared__ __align__(1024) char smem[];
    constexpr int NS = stages<KT>(), DC = DK / KS, SB = stage_bytes<DK, KT>();
    __shared__ uint64_t full[NS];
    __shared__ int dead_flag;
    using X = Exchange<DK, KT, KS>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const DeltaShape& s = a.s;
    const int groups = (a.l.slices + per - 1) / per;  // CTAs per sequence
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
    const int r0 = slice * 16 + g, r1 = r0 + 8;  // the lane's two value rows
    const bool ok0 = active && r0 < s.dv, ok1 = active && r1 < s.dv;
    const uint32_t ring = sm100::smem_u32(smem);

    if (chain) {
        const int col0 = part * DC;
        // S is kept times its scale: s_now, undone by s_inv
        float S[DC / 8][4], s_now = 1.0f, s_inv = 1.0f, norm = 0.0f;
#pragma unroll
        for (int j = 0; j < DC / 8; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int col = col0 + j * 8 + 2 * c4 + (x & 1);
                const bool ok = a.S_init && col < s.dk && (x < 2 ? ok0 : ok1);
                S[j][x] = ok ? a.S_init[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] : 0.0f;
            }
        // With |S| the slice's 2-norm:  |P| <= max |v| + max b |k| |S|,  |e| <= sum |T| |P|,  |S_next| <= b_end |S| + sum (|eta| D_end |k|) |e|
        // for every row.  |S| itself is summed beside the products, scaled, so that squares stay in range.
        float sk[4][4], squares0 = 0.0f, squares1 = 0.0f;  // S K^T of the next chunk
        uint32_t fh[2][4], fl[2][4];                       // fragments of two column tiles of S each: even and odd
        constexpr int TERMS = KT == 2 ? 3 : 2;             // products of an operand in two terms with a tile of the ring
        // a pair of columns of column tiles 2 kk, 2 kk + 1 of the warp's part of S into its fragment
        auto split_s = [&](int kk, int r) {
            const float (&y)[4] = S[2 * kk + (r >> 1)];
            const float y0 = y[2 * (r & 1)], y1 = y[2 * (r & 1) + 1];
            fma2(squares0, squares1, y0, y1, y0, y1, squares0, squares1);
            split(y0, y1, fh[kk & 1][r], fl[kk & 1][r]);
        };
        auto leave_s = [&](int kk, X& x) {  // for the outputs' warp
            const uint32_t (&h)[4] = fh[kk & 1], (&l)[4] = fl[kk & 1];
            x.s[0][part * (DC / 16) + kk][lane] = make_uint4(h[0], h[1], h[2], h[3]);
            x.s[1][part * (DC / 16) + kk][lane] = make_uint4(l[0], l[1], l[2], l[3]);
        };
        // the i-th two MMAs (of 2 TERMS) of those column tiles with a key tile
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
        auto hand = [&](X& x) {  // the warp's part of S K^T and of the norm: 32 times the largest of the lanes' sums bounds their sum
            const float y = 32.0f * warp_most(squares0 + squares1);
            if (KS == 1) {
                norm = y;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x.part[part][j][lane] = make_float4(sk[j][0], sk[j][1], sk[j][2], sk[j][3]);
                if (lane == 0) x.norm[part] = y;
            }
            if (lane == 0 && part == 0) x.s_inv = s_inv;
        };
        auto take = [&](const X& x) {  // all parts, in one order for all warps
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
        wait_phase(&full[0], 0, wait, 901);
        if (active) {
            float m = 0.0f;  // of the whole slice, so that all parts have one scale
            for (int col = c4; col < s.dk && a.S_init; col += 4) {
                if (ok0) m = fmaxf(m, fabsf(a.S_init[((size_t)n * s.dv + r0) * s.dk + col]));
                if (ok1) m = fmaxf(m, fabsf(a.S_init[((size_t)n * s.dv + r1) * s.dk + col]));
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
            if (SAVE) sm100::fence_proxy_async_smem();
        }
        __syncthreads();  // the values of chunk 0
        int st = 0, st_next = 1, phase_next = 0;
        for (int c = 0; c < nch; ++c) {
            const uint32_t ks = ring + st * SB, ts = ks + 2 * KT * 64 * DK, kn = ring + st_next * SB;
            const float* sc = reinterpret_cast<const float*>(smem + st * SB + 2 * KT * 64 * DK + 8192);
            const float* head = sc + kRecHead * 32;
            X& x = xb[c & 1];
            X& xn = xb[(c + 1) & 1];
            float e[4][4], uf = 0.0f, w_old = 0.0f, w_new = 0.0f;
            uint32_t wh[2][4], wl[2][4];
            const bool come = c + 1 == nch || probe_phase(&full[st_next], phase_next);
            if (active) {
                take(x);
                if (SAVE) {  // S K^T as it is, for the decays' gradients
                    const size_t at = ((size_t)n * nch + c) * a.l.slices + slice;
                    float4* dst = reinterpret_cast<float4*>(a.ws + a.l.sk) + at * 128;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (KS == 1 || part == (j >> 1)) dst[j * 32 + lane] = make_float4(sk[j][0], sk[j][1], sk[j][2], sk[j][3]);
                    if (lane == 0 && part == 0) reinterpret_cast<float*>(a.ws + a.l.c_inv)[at] = s_inv;
                }
                // T's blocks (the one above the diagonal is zero)
                uint32_t th[3][4], tl[3][4];  // (rows 0-15, k 0), (rows 16-31, k 0), (rows 16-31, k 1)
                ldsm4(th[0], addr_nk<32>(ts, 0, 0, lane)); ldsm4(th[1], addr_nk<32>(ts, 2, 0, lane)); ldsm4(th[2], addr_nk<32>(ts, 2, 1, lane));
                ldsm4(tl[0], addr_nk<32>(ts + 2048, 0, 0, lane)); ldsm4(tl[1], addr_nk<32>(ts + 2048, 2, 0, lane));
                ldsm4(tl[2], addr_nk<32>(ts + 2048, 2, 1, lane));
                const float bend = head[kHeadEnd];
                const float pb = fmaf(head[kHeadKn], norm, x.v_max), eb = pb * head[kHeadTsum];
                float f, q;
                pow2_bound(pb, f, q);
                // P, times its scale f
                float p[4][4];
                if (KT == 1) {
                    uint32_t v[2][4];
                    ldsm4_t(v[0], addr_tok(sm100::smem_u32(x.v), 0, lane));
                    ldsm4_t(v[1], addr_tok(sm100::smem_u32(x.v), 1, lane));
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const uint32_t w = v[j >> 1][(j & 1) * 2 + y];
                            mul2(p[j][2 * y], p[j][2 * y + 1], __uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u), f, f);
                        }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 v = x.v[KT == 1 ? 0 : j][lane];
                        mul2(p[j][0], p[j][1], v.x, v.y, f, f);
                        mul2(p[j][2], p[j][3], v.z, v.w, f, f);
                    }
                }
                const float fs = -scales(f, s_inv);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 bk = *reinterpret_cast<const float2*>(sc + kRecBk * 32 + j * 8 + 2 * c4);
                    float y0, y1;
                    mul2(y0, y1, bk.x, bk.y, fs, fs);
                    fma2(p[j][0], p[j][1], sk[j][0], sk[j][1], y0, y1, p[j][0], p[j][1]);
                    fma2(p[j][2], p[j][3], sk[j][2], sk[j][3], y0, y1, p[j][2], p[j][3]);
                }
                {
                    uint32_t h0[4], l0[4], h1[4], l1[4];
                    split_a(p[0], p[1], h0, l0);
                    mma0(e[0], h0, th[0][0], th[0][1]); mma0(e[1], h0, th[0][2], th[0][3]);
                    mma0(e[2], h0, th[1][0], th[1][1]); mma0(e[3], h0, th[1][2], th[1][3]);
                    split_a(p[2], p[3], h1, l1);
                    // the second terms' products apart: an MMA truncates the sum that it adds to
                    float t[4][4];
                    mma0(t[0], l0, th[0][0], th[0][1]); mma0(t[1], l0, th[0][2], th[0][3]);
                    mma0(t[2], l0, th[1][0], th[1][1]); mma0(t[3], l0, th[1][2], th[1][3]);
                    mma(e[2], h1, th[2][0], th[2][1]); mma(e[3], h1, th[2][2], th[2][3]);
                    mma(t[0], h0, tl[0][0], tl[0][1]); mma(t[1], h0, tl[0][2], tl[0][3]);
                    mma(t[2], h0, tl[1][0], tl[1][1]); mma(t[3], h0, tl[1][2], tl[1][3]);
                    mma(t[2], l1, th[2][0], th[2][1]); mma(t[3], l1, th[2][2], th[2][3]);
                    mma(t[2], h1, tl[2][0], tl[2][1]); mma(t[3], h1, tl[2][2], tl[2][3]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        add2(e[j][0], e[j][1], t[j][0], t[j][1]);
                        add2(e[j][2], e[j][3], t[j][2], t[j][3]);
                    }
                }
                // e times qe is the error itself.  It goes to the outputs' warp, eta D_end e into the state, each with a scale of its own;
                // the state moves to its next scale on the way
                const float qe = q * head[kHeadT];
                float pu, u_inv, fw, w_inv;
                pow2_bound(eb, pu, u_inv);
                pow2_bound(eb * head[kHeadWmax], fw, w_inv);
                uf = pu * qe;
                const float wf = scales(fw, qe), old_inv = s_inv;
                pow2_bound(fmaf(bend, norm, eb * head[kHeadWsum]), s_now, s_inv);
                w_old = scales(bend * old_inv, s_now);
                w_new = w_inv * s_now;
                if (lane == 0 && part == 0) x.u_inv = u_inv;
                float w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 we = *reinterpret_cast<const float2*>(sc + kRecW * 32 + j * 8 + 2 * c4);
                    float y0, y1;
                    mul2(y0, y1, we.x, we.y, wf, wf);
                    mul2(w[j][0], w[j][1], e[j][0], e[j][1], y0, y1);
                    mul2(w[j][2], w[j][3], e[j][2], e[j][3], y0, y1);
                }
                split_a(w[0], w[1], wh[0], wl[0]);
                split_a(w[2], w[3], wh[1], wl[1]);
            }
            if (!come) sm100::mbar_wait(&full[st_next], phase_next, wait, 901);
            if (active) {
                // S = b_end S + (D_end u) K, 32 columns at a time: the sum of the chunk apart from the state (the MMAs truncate what they add to),
                // then one rounding.  A piece's columns go on into the next chunk's S K^T while the next piece is summed.  (Behind the last
                // chunk that product is of whatever the ring holds, and unused.)
                // A warp issues in order, and an MMA that finds the pipe busy holds up what stands behind it: the arithmetic of a piece is cut into
                // twelve steps (a column tile of S, four times, and its fragments' pairs, eight times), with the MMAs in twos between
                // them.  Fragments are fetched a piece ahead of the products that they are for.
                constexpr int NJ = DC / 32;
                float y[2][4][4];
                uint32_t fs[2][2][KT][4], fk[2][2 * KT][4];
                auto load_s = [&](int j4) {
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int k = 0; k < KT; ++k) ldsm4_t(fs[kk][h][k], addr_kn<DK>(ks + k * 64 * DK, part * (DC / 8) + 4 * j4 + 2 * h, kk, lane));
                };
                auto sum = [&](float (&t)[4][4], int i) {  // the i-th two MMAs (of 4 TERMS)
                    const int kk = i / (2 * TERMS), term = i % (2 * TERMS) >> 1, h = i & 1;
                    const uint32_t (&w)[4] = term == 1 ? wl[kk] : wh[kk];
                    const uint32_t (&b)[4] = fs[kk][h][term == 2 ? KT - 1 : 0];
                    if (kk == 0 && term == 0) {
                        mma0(t[2 * h], w, b[0], b[1]);
                        mma0(t[2 * h + 1], w, b[2], b[3]);
                    } else {
                        mma(t[2 * h], w, b[0], b[1]);
                        mma(t[2 * h + 1], w, b[2], b[3]);
                    }
                };
                load_s(0);
                squares0 = squares1 = 0.0f;
                // e's fragments for the outputs, shared out between the parts; beside the first piece's sum
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
                    for (int i = 0; i < 2 * TERMS; ++i) sum(y[0], kk * 2 * TERMS + i);
                    if (KS > 1 && part != kk) continue;
#pragma unroll
                    for (int j = 2 * kk; j < 2 * kk + 2; ++j) {
                        mul2(e[j][0], e[j][1], e[j][0], e[j][1], uf, uf);
                        mul2(e[j][2], e[j][3], e[j][2], e[j][3], uf, uf);
                    }
                    uint32_t hi[4], lo[4];
                    split_a(e[2 * kk], e[2 * kk + 1], hi, lo);
                    x.u[0][kk][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    x.u[1][kk][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                if (NJ > 1) load_s(1);
                load_k(kn, 0, fk[0]);
#pragma unroll
                for (int j4 = 0; j4 < NJ; ++j4) {
                    // the MMAs beside this piece: the odd column tiles of the one before with the keys, the next one's sum, the even tiles of this one
                    const int before = j4 > 0 ? 2 * TERMS : 0, next = j4 + 1 < NJ ? 4 * TERMS : 0, all = before + next + 2 * TERMS;
                    auto upto = [&](int m) {  // how many behind step m; the even tiles' fragments are whole behind step 5
                        const int most = m < 5 ? before + next : all;
                        return (m + 1) * all / 12 < most ? (m + 1) * all / 12 : most;
                    };
                    auto issue = [&](int i) {
                        if (i < before) times_k(2 * j4 - 1, i, false, fk[1]);
                        else if (i < before + next) sum(y[(j4 + 1) & 1], i - before);
                        else times_k(2 * j4, i - before - next, j4 == 0, fk[0]);
                        if (i + 1 == before || (i == 0 && before == 0)) load_k(kn, 2 * j4 + 1, fk[1]);
                        if (next > 0 && i + 1 == before + next && j4 + 2 < NJ) load_s(j4 + 2);
                    };
#pragma unroll
                    for (int m = 0; m < 12; ++m) {
                        if (m == 0 || m == 1 || m == 6 || m == 7) {  // a column tile of S
                            const int i = m < 2 ? m : m - 4;
                            float (&d)[4] = S[4 * j4 + i];
                            const float (&t)[4] = y[j4 & 1][i];
#pragma unroll
                            for (int z = 0; z < 4; z += 2) {
                                float m0, m1;
                                mul2(m0, m1, d[z], d[z + 1], w_old, w_old);
                                fma2(d[z], d[z + 1], t[z], t[z + 1], w_new, w_new, m0, m1);
                            }
                        } else {
                            const int r = m < 6 ? m - 2 : m - 8;
                            split_s(2 * j4 + (m < 6 ? 0 : 1), r);
                            if (r == 3) leave_s(2 * j4 + (m < 6 ? 0 : 1), xn);
                        }
#pragma unroll
                        for (int i = upto(m - 1); i < upto(m); ++i) issue(i);
                    }
                    if (j4 + 1 < NJ) load_k(kn, 2 * j4 + 2, fk[0]);
                }
#pragma unroll
                for (int i = 0; i < 2 * TERMS; ++i) times_k(2 * NJ - 1, i, false, fk[1]);
                hand(xn);
                if (SAVE) sm100::fence_proxy_async_smem();  // the outputs' warp has the fragments copied from there
            }
            st = st_next;
            if (++st_next == NS) { st_next = 0; phase_next ^= 1; }
            __syncthreads();
        }
        if (active) {
            if (a.S_final) {
#pragma unroll
                for (int j = 0; j < DC / 8; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int col = col0 + j * 8 + 2 * c4 + (x & 1);
                        if (col < s.dk && (x < 2 ? ok0 : ok1)) a.S_final[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] = S[j][x] * s_inv;
                    }
            }
        }
        return;
    }

    // ---- the outputs' warp of a slice
    const char* qk_src = a.ws + a.l.qk + (size_t)nk * nch * a.l.qk_bytes;
    const char* rec_src = a.ws + a.l.rec + (size_t)n * nch * a.l.rec_bytes;
    const bool fetches = mine == 0 && lane == 0;
    auto fetch = [&](int c, int st) {
        const uint32_t dst = ring + st * SB;
        uint64_t* bar = &full[st];
        sm100::mbar_expect_tx(bar, SB);
        bulk_copy(dst, qk_src + (size_t)c * a.l.qk_bytes, 2 * KT * 64 * DK, bar);
        bulk_copy(dst + 2 * KT * 64 * DK, rec_src + (size_t)c * a.l.rec_bytes, kDeltaRecBytes, bar);
    };
    if (fetches)
        for (int c = 0; c < NS && c < nch; ++c) fetch(c, c);
    __syncwarp();
    const IO* v = reinterpret_cast<const IO*>(a.v) + (size_t)n * s.L * s.dv + slice * 16;
    IO* o = a.o ? reinterpret_cast<IO*>(a.o) + (size_t)n * s.L * s.dv + slice * 16 : nullptr;
    const int rows = active ? min(16, s.dv - slice * 16) : 0;  // value rows of the slice
    // The values of a chunk: bf16, lane = token, its 16 rows in two pieces; fp32, in fragment order.  Asynchronous copies, so that nothing
    // that the warp waits for on the way to the outputs waits for them (rows of odd widths go through registers)
    uint32_t odd[8];
    auto load_v = [&](int c) {
        X& x = xb[c & 1];
        if (KT == 1) {
            const int t = c * kDeltaChunk + lane;
            const IO* p = v + (size_t)t * s.dv;
            const int here = t < s.L ? rows : 0;
            if (vec) {
                const uint32_t tile = sm100::smem_u32(x.v);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tile + tok_at(lane, i)), "l"(here > 8 * i ? p + 8 * i : v), "r"(here > 8 * i ? 16 : 0) : "memory");
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t y = 2 * i < here ? reinterpret_cast<const uint16_t*>(p)[2 * i] : 0u;
                    const uint32_t z = 2 * i + 1 < here ? reinterpret_cast<const uint16_t*>(p)[2 * i + 1] : 0u;
                    odd[i] = y | z << 16;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (i & 1), r = g + (i < 2 ? 0 : 8);
                    const bool ok = t < s.L && r < rows;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(sm100::smem_u32(&x.v[KT == 1 ? 0 : j][lane]) + 4 * i), "l"(ok ? v + (size_t)t * s.dv + r : v), "r"(ok ? 4 : 0) : "memory");
                }
        }
    };
    auto hand_v = [&](int c) {  // the copies have come; a bound on the values
        X& x = xb[c & 1];
        float m = 0.0f;
        if (KT == 1) {
            char* tile = reinterpret_cast<char*>(x.v);
            if (!vec) {
                *reinterpret_cast<uint4*>(tile + tok_at(lane, 0)) = make_uint4(odd[0], odd[1], odd[2], odd[3]);
                *reinterpret_cast<uint4*>(tile + tok_at(lane, 1)) = make_uint4(odd[4], odd[5], odd[6], odd[7]);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            const uint4 y = *reinterpret_cast<const uint4*>(tile + tok_at(lane, 0)), z = *reinterpret_cast<const uint4*>(tile + tok_at(lane, 1));
            uint32_t top = 0;  // largest magnitude on the bits: both halves of a word at a time
            const uint32_t w[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
            m = __uint_as_float(max(top << 16, top & 0xffff0000u));
        } else {
            asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 y = x.v[KT == 1 ? 0 : j][lane];
                m = fmaxf(m, fmaxf(fmaxf(fabsf(y.x), fabsf(y.y)), fmaxf(fabsf(y.z), fabsf(y.w))));
            }
        }
        m = warp_most(m);
        if (lane == 0) x.v_max = m;
    };
    auto product = [&](int c, int st, float (&sq)[4][4]) {  // S Q^T, in S's scale
        const uint32_t qs = ring + st * SB + KT * 64 * DK;
        const X& x = xb[c & 1];
        uint4 f[2][2];
        float sl[4][4] = {};  // the second terms' products apart: an MMA truncates the sum that it adds to
        uint32_t b[2][2][KT][4];
        auto load = [&](int kk) {
#pragma unroll
            for (int t = 0; t < 2; ++t) f[kk & 1][t] = x.s[t][kk][lane];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < KT; ++t) ldsm4(b[kk & 1][h][t], addr_nk<DK>(qs + t * 64 * DK, 2 * h, kk, lane));
        };
        load(0);
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            if (kk + 1 < DK / 16) load(kk + 1);
            const uint4 h4 = f[kk & 1][0], l4 = f[kk & 1][1];
            const uint32_t hi[4] = {h4.x, h4.y, h4.z, h4.w}, lo[4] = {l4.x, l4.y, l4.z, l4.w};
            const uint32_t (&q)[2][KT][4] = b[kk & 1];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (kk == 0) { mma0(sq[2 * h], hi, q[h][0][0], q[h][0][1]); mma0(sq[2 * h + 1], hi, q[h][0][2], q[h][0][3]); }
                else { mma(sq[2 * h], hi, q[h][0][0], q[h][0][1]); mma(sq[2 * h + 1], hi, q[h][0][2], q[h][0][3]); }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) { mma(sl[2 * h], lo, q[h][0][0], q[h][0][1]); mma(sl[2 * h + 1], lo, q[h][0][2], q[h][0][3]); }
            if (KT == 2)
#pragma unroll
                for (int h = 0; h < 2; ++h) { mma(sl[2 * h], hi, q[h][KT - 1][0], q[h][KT - 1][1]); mma(sl[2 * h + 1], hi, q[h][KT - 1][2], q[h][KT - 1][3]); }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int y = 0; y < 4; ++y) sq[j][y] += sl[j][y];
    };
    auto finish = [&](int c, int st, const float (&sq)[4][4], float s_inv) {  // O = b S Q^T + e (A eta)^T
        const uint32_t as = ring + st * SB + 2 * KT * 64 * DK + 4096;
        const float* sc = reinterpret_cast<const float*>(smem + st * SB + 2 * KT * 64 * DK + 8192);
        X& x = xb[c & 1];
        float in[4][4] = {}, il[4][4] = {};
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint4 h4 = x.u[0][kk][lane], l4 = x.u[1][kk][lane];
            const uint32_t hi[4] = {h4.x, h4.y, h4.z, h4.w}, lo[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
            for (int h = kk; h < 2; ++h) {
                uint32_t bh[4], bl[4];
                ldsm4(bh, addr_nk<32>(as, 2 * h, kk, lane));
                mma(in[2 * h], hi, bh[0], bh[1]); mma(in[2 * h + 1], hi, bh[2], bh[3]);
                ldsm4(bl, addr_nk<32>(as + 2048, 2 * h, kk, lane));
                mma(il[2 * h], lo, bh[0], bh[1]); mma(il[2 * h + 1], lo, bh[2], bh[3]);
                mma(il[2 * h], hi, bl[0], bl[1]); mma(il[2 * h + 1], hi, bl[2], bl[3]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int y = 0; y < 4; ++y) in[j][y] += il[j][y];
        const float q = x.u_inv * sc[kRecHead * 32 + kHeadA];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 bq = *reinterpret_cast<const float2*>(sc + kRecBq * 32 + j * 8 + 2 * c4);
            float y0, y1;
            mul2(y0, y1, bq.x, bq.y, s_inv, s_inv);
#pragma unroll
            for (int z = 0; z < 4; z += 2) {
                mul2(in[j][z], in[j][z + 1], in[j][z], in[j][z + 1], q, q);
                fma2(in[j][z], in[j][z + 1], sq[j][z], sq[j][z + 1], y0, y1, in[j][z], in[j][z + 1]);
            }
        }
        if (SAVE) {
            float4* dst = reinterpret_cast<float4*>(a.ws + a.l.sq) + (((size_t)n * nch + c) * a.l.slices + slice) * 128;
#pragma unroll
            for (int j = 0; j < 4; ++j) dst[j * 32 + lane] = make_float4(sq[j][0], sq[j][1], sq[j][2], sq[j][3]);
        }
        if (!o) return;
        if (KT == 1) {  // through shared memory to lane = token
            const uint32_t tile = sm100::smem_u32(x.o);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                stsm4_t(addr_tok(tile, h, lane), pack_bf16(in[2 * h][0], in[2 * h][1]), pack_bf16(in[2 * h][2], in[2 * h][3]),
                        pack_bf16(in[2 * h + 1][0], in[2 * h + 1][1]), pack_bf16(in[2 * h + 1][2], in[2 * h + 1][3]));
            __syncwarp();
            const int t = c * kDeltaChunk + lane;
            const char* row = reinterpret_cast<const char*>(x.o);
            const uint4 y0 = *reinterpret_cast<const uint4*>(row + tok_at(lane, 0)), y1 = *reinterpret_cast<const uint4*>(row + tok_at(lane, 1));
            if (t >= s.L) return;
            IO* p = o + (size_t)t * s.dv;
            if (vec) {
                reinterpret_cast<uint4*>(p)[0] = y0;
                if (rows > 8) reinterpret_cast<uint4*>(p)[1] = y1;
            } else {
                const uint32_t w[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (2 * i < rows) reinterpret_cast<uint16_t*>(p)[2 * i] = (uint16_t)w[i];
                    if (2 * i + 1 < rows) reinterpret_cast<uint16_t*>(p)[2 * i + 1] = (uint16_t)(w[i] >> 16);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int t = c * kDeltaChunk + j * 8 + 2 * c4 + (y & 1), r = g + (y < 2 ? 0 : 8);
                    if (t < s.L && r < rows) o[(size_t)t * s.dv + r] = from_f32<IO>(in[j][y]);
                }
        }
    };
    // what the reverse pass reads of S and e: their fragments as they lie in shared memory
    auto save_s = [&](int slot, const X& x) {
        if (lane != 0) return;
        const size_t at = ((size_t)n * a.l.nblk + slot) * a.l.slices + slice;
        bulk_store(a.ws + a.l.S + at * a.l.state_bytes, sm100::smem_u32(x.s[0]), (uint32_t)a.l.state_bytes);
        bulk_store(a.ws + a.l.S_lo + at * a.l.state_bytes, sm100::smem_u32(x.s[1]), (uint32_t)a.l.state_bytes);
        reinterpret_cast<float*>(a.ws + a.l.s_inv)[at] = x.s_inv;
    };
    auto save_e = [&](int c, const X& x) {
        if (lane != 0) return;
        const size_t at = ((size_t)n * nch + c) * a.l.slices + slice;
        bulk_store(a.ws + a.l.e + at * 2048, sm100::smem_u32(x.u), 2048);
        reinterpret_cast<float*>(a.ws + a.l.e_inv)[at] = x.u_inv;
    };
    load_v(0);
    hand_v(0);
    __syncthreads();
    float sq[4][4], s_inv = 1.0f;
    int st = 0, phase = 0;
    for (int i = 0; i <= nch; ++i) {
        if (i + 1 < nch) load_v(i + 1);  // the chain reads chunk i's
        if (SAVE && active) {
            if (i > 0) save_e(i - 1, xb[(i - 1) & 1]);
            if (i < nch && (i & 1) == 0) save_s(i >> 1, xb[i & 1]);
            bulk_store_commit();
        }
        if (active && i > 0) finish(i - 1, st == 0 ? NS - 1 : st - 1, sq, s_inv);
        if (i < nch) {
            wait_phase(&full[st], phase, wait, 903);
            if (active) {
                product(i, st, sq);
                s_inv = xb[i & 1].s_inv;
            }
            if (i + 1 < nch) hand_v(i + 1);
            if (SAVE) bulk_store_read();  // the chain may write there again
            __syncthreads();  // chunk i is through the chain, chunk i - 1 through here
        }
        if (fetches && i > 0 && i - 1 + NS < nch) fetch(i - 1 + NS, st == 0 ? NS - 1 : st - 1);
        __syncwarp();
        if (++st == NS) { st = 0; phase ^= 1; }
    }
    if (SAVE) bulk_store_done();
}

template <typename IO, int DK, int KT, int KS, bool SAVE> int launch(const DeltaArgs& a, int per, cudaStream_t st) {
    auto kernel = delta_fwd_kernel<IO, DK, KT, KS, SAVE>;
    const int bytes = fwd_smem<DK, KT, KS>(per);
    cudaError_t e = allow_shared_memory<delta_fwd_kernel<IO, DK, KT, KS, SAVE>>();
    if (e != cudaSuccess) return (int)e;
    const unsigned grid = (unsigned)(a.l.N * ((a.l.slices + per - 1) / per));
    const bool vec = a.s.dv % 8 == 0 && (reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.o)) % 16 == 0;
    kernel<<<grid, per * (KS + 1) * 32, bytes, st>>>(a, per, vec);
    return (int)cudaGetLastError();
}

template <typename IO, int DK, int KT, bool SAVE> int dispatch(const DeltaArgs& a, cudaStream_t st) {
    constexpr int most = KT == 1 ? 4 : 2;
    static_assert(fwd_smem<DK, KT, 1>(most) <= kMostSharedMemory && (KT == 1 || fwd_smem<DK, KT, DK / 32>(1) <= kMostSharedMemory), "shared memory");
    // fp32, few slices, as many as SMs at most: one per CTA, its columns over DK / 32 warps.  Calls of 2048 tokens, us: 16 heads of 128 x 128: 175, with a warp per
    // slice 188; 12 of 64 x 64: 107 and 115.  With bf16, whose chain has two products where fp32 has three, the outputs' warp would hold up the chain's: 111 and
    // 103, 76.5 and 76.4.  More slices than SMs: a chain per warp, and slices of a sequence share the tiles that they fetch, as long as 96 CTAs are
    // left.  bf16, us: forward and reverse pass, 8 x 12 x 2048 tokens, 64 x 64: 4 slices per CTA 604, 2: 679, 1: 734, one over two warps 731.  Forward
    // alone, 128 x 128, 16 heads x 4096 tokens: B = 4: 4 slices 344, 2: 427; B = 2: 2 slices 222, 4: 302; B = 1: 1 slice 201, 4: 282.  fp32 tiles leave room for two.
    if constexpr (KT == 2)
        if (a.l.N * a.l.slices <= 148) return launch<IO, DK, KT, DK / 32, SAVE>(a, 1, st);
    return launch<IO, DK, KT, 1, SAVE>(a, slices_per_cta(a.l, most), st);
}

template <typename IO, int DK, int KT> int either(const DeltaArgs& a, cudaStream_t st) {
    return a.save ? dispatch<IO, DK, KT, true>(a, st) : dispatch<IO, DK, KT, false>(a, st);
}

}  // namespace

int delta_fwd_launch(const DeltaArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.s.f32) return a.l.DK == 64 ? either<float, 64, 2>(a, st) : either<float, 128, 2>(a, st);
    return a.l.DK == 64 ? either<__nv_bfloat16, 64, 1>(a, st) : either<__nv_bfloat16, 128, 1>(a, st);
}

}  // namespace e2ttt
