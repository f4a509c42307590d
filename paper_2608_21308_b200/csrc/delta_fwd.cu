// Gated delta rule, the walk over the chunks.  A warp owns 16 value rows of one sequence's state: the slice [16, dk] stays in its registers
// (64 of them at dk = 128) from the first token to the last, and the slices of a sequence never meet but for the tiles that they share.
// Per chunk of 32 tokens, rows = value rows:  P = V - b S K^T,  e = P T^T,  O = b S Q^T + u A^T,  S = b_end S + (D_end u) K.
// Each product's result is the next one's A operand in place.  The chunk's tiles (queries, keys, T, A, scalars; written by
// delta_prep.cu) arrive by bulk copies, several chunks ahead.
// The chain P, e, S is what a chunk waits for; a second warp per slice, a chunk behind, does what hangs off it: O from the state's and u's fragments
// (which the first one leaves in shared memory), and the values' loads and the outputs' stores.  One barrier a chunk.
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

template <int DK, int KT> constexpr int stage_bytes() { return 2 * KT * 64 * DK + kDeltaRecBytes; }
template <int KT> constexpr int stages() { return KT == 1 ? 4 : 3; }

// what the two warps of a slice hand over, a buffer per parity of the chunk: fragments of S and u (a second term each with PREC), the scales
// that they carry, and the values of the next chunk, all in fragment order
template <int DK, bool PREC> struct alignas(16) Exchange {
    uint4 s[PREC ? 2 : 1][DK / 16][32];
    uint4 u[PREC ? 2 : 1][2][32];
    float2 s_inv[32], u_inv[32], v_max[32];
    float4 v[4][32];
};

template <int DK, int KT, bool PREC> constexpr int fwd_smem(int warps) {
    return stages<KT>() * stage_bytes<DK, KT>() + 2 * warps * (int)sizeof(Exchange<DK, PREC>);
}

// PREC: both terms in the outputs' products as well (fp32 outputs, or outputs that the reverse pass needs in 32 bits).  Without it an output
// is off by 2^-12 of its terms before it is rounded to bf16's 2^-9.
template <typename IO, int DK, int KT, bool PREC>
__global__ void __launch_bounds__(256) delta_fwd_kernel(const DeltaArgs a, const int warps) {
    extern __shared__ __align__(1024) char smem[];
    constexpr int NS = stages<KT>(), SB = stage_bytes<DK, KT>();
    __shared__ uint64_t full[NS];
    __shared__ int dead_flag;
    using X = Exchange<DK, PREC>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const DeltaShape& s = a.s;
    const int groups = (a.l.slices + warps - 1) / warps;  // CTAs per sequence
    const int64_t n = blockIdx.x / groups, nk = (n / s.H) * s.Hk + (n % s.H) / (s.H / s.Hk);
    const bool chain = warp < warps;
    const int mine = chain ? warp : warp - warps;
    const int slice = (int)(blockIdx.x % groups) * warps + mine;
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

    if (chain) {
        float S[DK / 8][4];
#pragma unroll
        for (int j = 0; j < DK / 8; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int col = j * 8 + 2 * c4 + (x & 1);
                const bool ok = a.S_init && col < s.dk && (x < 2 ? ok0 : ok1);
                S[j][x] = ok ? a.S_init[((size_t)n * s.dv + (x < 2 ? r0 : r1)) * s.dk + col] : 0.0f;
            }
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
        // Scales come from bounds that are known before the values are (the chain waits for no maximum): with |S| the 2-norm of a row,
        //   |P| <= max |v| + max b |k| |S|,  |e| <= sum |T| |P|,  |S_next| <= b_end |S| + sum (|eta| D_end |k|) |e|.
        float sk[4][4], sl[4][4];                     // S K^T of the next chunk, first and second term
        float n0 = 0.0f, n1 = 0.0f, i0, i1, s0, s1;   // row norms of S; its scales
        // column tiles 2 kk, 2 kk + 1 of S: fragments to the second warp and into S K^T
        auto with_k = [&](uint32_t ks, int kk, X& x, const uint32_t (&b)[2 * KT][4]) {
            uint32_t hi[4], lo[4];
            float (&y)[4] = S[2 * kk], (&z)[4] = S[2 * kk + 1];
            const float y0 = y[0] * s0, y1 = y[1] * s0, y2 = y[2] * s1, y3 = y[3] * s1, z0 = z[0] * s0, z1 = z[1] * s0, z2 = z[2] * s1, z3 = z[3] * s1;
            n0 = fmaf(y0, y0, n0); n0 = fmaf(z0, z0, n0); n1 = fmaf(y2, y2, n1); n1 = fmaf(z2, z2, n1);
            n0 = fmaf(y1, y1, n0); n0 = fmaf(z1, z1, n0); n1 = fmaf(y3, y3, n1); n1 = fmaf(z3, z3, n1);
            split(y0, y1, hi[0], lo[0]); split(y2, y3, hi[1], lo[1]); split(z0, z1, hi[2], lo[2]); split(z2, z3, hi[3], lo[3]);
            x.s[0][kk][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            if (PREC) x.s[PREC ? 1 : 0][kk][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            mma(sk[0], hi, b[0][0], b[0][1]); mma(sk[1], hi, b[0][2], b[0][3]);
            mma(sk[2], hi, b[1][0], b[1][1]); mma(sk[3], hi, b[1][2], b[1][3]);
            mma(sl[0], lo, b[0][0], b[0][1]); mma(sl[1], lo, b[0][2], b[0][3]);
            mma(sl[2], lo, b[1][0], b[1][1]); mma(sl[3], lo, b[1][2], b[1][3]);
            if (KT == 2) {
                constexpr int f = KT == 2 ? 2 : 0, h = KT == 2 ? 3 : 0;
                mma(sl[0], hi, b[f][0], b[f][1]); mma(sl[1], hi, b[f][2], b[f][3]);
                mma(sl[2], hi, b[h][0], b[h][1]); mma(sl[3], hi, b[h][2], b[h][3]);
            }
        };
        auto load_k = [&](uint32_t ks, int kk, uint32_t (&b)[2 * KT][4]) {
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                ldsm4(b[2 * t], addr_nk<DK>(ks + t * 64 * DK, 0, kk, lane));
                ldsm4(b[2 * t + 1], addr_nk<DK>(ks + t * 64 * DK, 2, kk, lane));
            }
        };
        auto begin = [&](X& x, float bound0, float bound1) {
            pow2_bound(bound0, s0, i0);
            pow2_bound(bound1, s1, i1);
            x.s_inv[lane] = make_float2(i0, i1);
            n0 = n1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) sk[j][y] = sl[j][y] = 0.0f;
        };
        auto norms = [&]() {
            n0 = sqrtf(quad_sum(n0)) * i0;
            n1 = sqrtf(quad_sum(n1)) * i1;
        };
        const uint32_t ring = sm100::smem_u32(smem);
        sm100::mbar_wait(&full[0], 0, wait, 901);
        if (active) {
            float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
            for (int j = 0; j < DK / 8; ++j) {
                m0 = fmaxf(m0, fmaxf(fabsf(S[j][0]), fabsf(S[j][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(S[j][2]), fabsf(S[j][3])));
            }
            begin(xb[0], quad_max(m0), quad_max(m1));
#pragma unroll
            for (int kk = 0; kk < DK / 16; ++kk) {
                uint32_t b[2 * KT][4];
                load_k(ring, kk, b);
                with_k(ring, kk, xb[0], b);
            }
            norms();
        }
        __syncthreads();  // the values of chunk 0
        for (int c = 0; c < nch; ++c) {
            const int st = c % NS;
            const uint32_t ks = ring + st * SB, ts = ks + 2 * KT * 64 * DK, kn = ring + (c + 1) % NS * SB;
            const float* sc = reinterpret_cast<const float*>(smem + st * SB + 2 * KT * 64 * DK + 8192);
            const float* head = sc + kRecHead * 32;
            X& x = xb[c & 1];
            X& xn = xb[(c + 1) & 1];
            float u[4][4], e[4][4], w0i, w1i;
            uint32_t wh[2][4], wl[2][4];
            float p0, p1, q0, q1, bend = 0.0f;
            if (active) {
                if (a.save && (c & 1) == 0) save_state(c >> 1);
                // T's blocks (the one above the diagonal is zero)
                uint32_t th[3][4], tl[3][4];  // (rows 0-15, k 0), (rows 16-31, k 0), (rows 16-31, k 1)
                ldsm4(th[0], addr_nk<32>(ts, 0, 0, lane)); ldsm4(th[1], addr_nk<32>(ts, 2, 0, lane)); ldsm4(th[2], addr_nk<32>(ts, 2, 1, lane));
                ldsm4(tl[0], addr_nk<32>(ts + 2048, 0, 0, lane)); ldsm4(tl[1], addr_nk<32>(ts + 2048, 2, 0, lane));
                ldsm4(tl[2], addr_nk<32>(ts + 2048, 2, 1, lane));
                bend = head[kHeadEnd];
                const float2 vm = x.v_max[lane];
                const float pb0 = fmaf(head[kHeadKn], n0, vm.x), pb1 = fmaf(head[kHeadKn], n1, vm.y);
                const float eb0 = pb0 * head[kHeadTsum], eb1 = pb1 * head[kHeadTsum];
                float f0, f1;
                pow2_bound(pb0, f0, q0);
                pow2_bound(pb1, f1, q1);
                float p[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 bk = *reinterpret_cast<const float2*>(sc + kRecBk * 32 + j * 8 + 2 * c4);
                    const float4 v = x.v[j][lane];
                    p[j][0] = fmaf(-(sk[j][0] + sl[j][0]) * i0, bk.x, v.x); p[j][1] = fmaf(-(sk[j][1] + sl[j][1]) * i0, bk.y, v.y);
                    p[j][2] = fmaf(-(sk[j][2] + sl[j][2]) * i1, bk.x, v.z); p[j][3] = fmaf(-(sk[j][3] + sl[j][3]) * i1, bk.y, v.w);
#pragma unroll
                    for (int y = 0; y < 4; ++y) e[j][y] = 0.0f;
                }
                {
                    uint32_t h0[4], l0[4], h1[4], l1[4];
                    to_a(p[0], p[1], f0, f1, h0, l0);
                    to_a(p[2], p[3], f0, f1, h1, l1);
                    float f[4][4] = {};
                    mma(e[0], h0, th[0][0], th[0][1]); mma(e[1], h0, th[0][2], th[0][3]);
                    mma(e[2], h0, th[1][0], th[1][1]); mma(e[3], h0, th[1][2], th[1][3]);
                    mma(f[0], l0, th[0][0], th[0][1]); mma(f[1], l0, th[0][2], th[0][3]);
                    mma(f[2], l0, th[1][0], th[1][1]); mma(f[3], l0, th[1][2], th[1][3]);
                    mma(e[2], h1, th[2][0], th[2][1]); mma(e[3], h1, th[2][2], th[2][3]);
                    mma(f[0], h0, tl[0][0], tl[0][1]); mma(f[1], h0, tl[0][2], tl[0][3]);
                    mma(f[2], h0, tl[1][0], tl[1][1]); mma(f[3], h0, tl[1][2], tl[1][3]);
                    mma(e[2], l1, th[2][0], th[2][1]); mma(e[3], l1, th[2][2], th[2][3]);
                    mma(f[2], h1, tl[2][0], tl[2][1]); mma(f[3], h1, tl[2][2], tl[2][3]);
                    q0 *= head[kHeadT]; q1 *= head[kHeadT];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        e[j][0] = (e[j][0] + f[j][0]) * q0; e[j][1] = (e[j][1] + f[j][1]) * q0;
                        e[j][2] = (e[j][2] + f[j][2]) * q1; e[j][3] = (e[j][3] + f[j][3]) * q1;
                    }
                }
                // u = eta e for the outputs, D_end u for the state: each with scales of its own
                pow2_bound(eb0 * head[kHeadUmax], p0, q0);
                pow2_bound(eb1 * head[kHeadUmax], p1, q1);
                pow2_bound(eb0 * head[kHeadWmax], f0, w0i);
                pow2_bound(eb1 * head[kHeadWmax], f1, w1i);
                float w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 et = *reinterpret_cast<const float2*>(sc + kRecEta * 32 + j * 8 + 2 * c4);
                    const float2 de = *reinterpret_cast<const float2*>(sc + kRecDend * 32 + j * 8 + 2 * c4);
                    u[j][0] = e[j][0] * et.x; u[j][1] = e[j][1] * et.y; u[j][2] = e[j][2] * et.x; u[j][3] = e[j][3] * et.y;
                    w[j][0] = u[j][0] * de.x; w[j][1] = u[j][1] * de.y; w[j][2] = u[j][2] * de.x; w[j][3] = u[j][3] * de.y;
                }
                to_a(w[0], w[1], f0, f1, wh[0], wl[0]);
                to_a(w[2], w[3], f0, f1, wh[1], wl[1]);
                begin(xn, fmaf(bend, n0, eb0 * head[kHeadWsum]), fmaf(bend, n1, eb1 * head[kHeadWsum]));
            }
            if (c + 1 < nch) sm100::mbar_wait(&full[(c + 1) % NS], ((c + 1) / NS) & 1, wait, 901);
            if (active) {
                // S = b_end S + (D_end u) K, 32 columns at a time: the sum of the chunk apart from the state (the MMAs truncate what they add to),
                // then one rounding.  A piece's columns go on into the next chunk's S K^T while the next piece is summed.  (Behind the last
                // chunk that product is of whatever the ring holds, and unused.)
                float y[2][4][4];
                auto sum = [&](int j4, float (&t)[4][4]) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int z = 0; z < 4; ++z) t[i][z] = 0.0f;
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        uint32_t b[2][KT][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int k = 0; k < KT; ++k) ldsm4_t(b[h][k], addr_kn<DK>(ks + k * 64 * DK, 4 * j4 + 2 * h, kk, lane));
#pragma unroll
                        for (int h = 0; h < 2; ++h) { mma(t[2 * h], wh[kk], b[h][0][0], b[h][0][1]); mma(t[2 * h + 1], wh[kk], b[h][0][2], b[h][0][3]); }
#pragma unroll
                        for (int h = 0; h < 2; ++h) { mma(t[2 * h], wl[kk], b[h][0][0], b[h][0][1]); mma(t[2 * h + 1], wl[kk], b[h][0][2], b[h][0][3]); }
                        if (KT == 2)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                mma(t[2 * h], wh[kk], b[h][KT - 1][0], b[h][KT - 1][1]);
                                mma(t[2 * h + 1], wh[kk], b[h][KT - 1][2], b[h][KT - 1][3]);
                            }
                    }
                };
                sum(0, y[0]);
#pragma unroll
                for (int j4 = 0; j4 < DK / 32; ++j4) {
                    if (j4 + 1 < DK / 32) sum(j4 + 1, y[(j4 + 1) & 1]);
                    uint32_t b0[2 * KT][4], b1[2 * KT][4];
                    load_k(kn, 2 * j4, b0);
                    load_k(kn, 2 * j4 + 1, b1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float (&d)[4] = S[4 * j4 + i];
                        const float (&t)[4] = y[j4 & 1][i];
                        d[0] = fmaf(t[0], w0i, bend * d[0]); d[1] = fmaf(t[1], w0i, bend * d[1]);
                        d[2] = fmaf(t[2], w1i, bend * d[2]); d[3] = fmaf(t[3], w1i, bend * d[3]);
                    }
                    with_k(kn, 2 * j4, xn, b0);
                    with_k(kn, 2 * j4 + 1, xn, b1);
                }
                // u's fragments for the outputs
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    uint32_t hi[4], lo[4];
                    to_a(u[2 * kk], u[2 * kk + 1], p0, p1, hi, lo);
                    x.u[0][kk][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    if (PREC) x.u[PREC ? 1 : 0][kk][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                x.u_inv[lane] = make_float2(q0, q1);
                norms();
                if (a.save) {
                    float m = 0.0f;
                    float* dst = reinterpret_cast<float*>(a.ws + a.l.e) + ((size_t)n * nch + c) * a.l.dvp * kDeltaChunk;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        *reinterpret_cast<float2*>(dst + r0 * kDeltaChunk + j * 8 + 2 * c4) = make_float2(e[j][0], e[j][1]);
                        *reinterpret_cast<float2*>(dst + r1 * kDeltaChunk + j * 8 + 2 * c4) = make_float2(e[j][2], e[j][3]);
                        m = fmaxf(m, fmaxf(fmaxf(fabsf(u[j][0]), fabsf(u[j][1])), fmaxf(fabsf(u[j][2]), fabsf(u[j][3]))));
                    }
                    m = warp_max(m);
                    if (lane == 0) reinterpret_cast<float*>(a.ws + a.l.max_u)[((size_t)n * nch + c) * a.l.slices + slice] = m;
                }
            }
            __syncthreads();
        }
        if (active) {
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
        return;
    }

    // ---- the second warp of a slice
    const char* qk_src = a.ws + a.l.qk + (size_t)nk * nch * a.l.qk_bytes;
    const char* rec_src = a.ws + a.l.rec + (size_t)n * nch * a.l.rec_bytes;
    const bool fetches = mine == 0 && lane == 0;
    auto fetch = [&](int c) {
        const uint32_t dst = sm100::smem_u32(smem) + (c % NS) * SB;
        uint64_t* bar = &full[c % NS];
        sm100::mbar_expect_tx(bar, SB);
        bulk_copy(dst, qk_src + (size_t)c * a.l.qk_bytes, 2 * KT * 64 * DK, bar);
        bulk_copy(dst + 2 * KT * 64 * DK, rec_src + (size_t)c * a.l.rec_bytes, kDeltaRecBytes, bar);
    };
    if (fetches)
        for (int c = 0; c < NS && c < nch; ++c) fetch(c);
    __syncwarp();
    const IO* v = reinterpret_cast<const IO*>(a.v) + (size_t)n * s.L * s.dv;
    IO* o = a.o ? reinterpret_cast<IO*>(a.o) + (size_t)n * s.L * s.dv : nullptr;
    IO vn[4][4];
    auto load_v = [&](int c) {
        const IO* p = v + ((size_t)c * kDeltaChunk + 2 * c4) * s.dv + r0;
        const int left = s.L - c * kDeltaChunk - 2 * c4;  // tokens from the lane's first one on
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = j * 8 + (i & 1);
                vn[j][i] = (t < left && (i < 2 ? ok0 : ok1)) ? p[(size_t)t * s.dv + (i < 2 ? 0 : 8)] : IO(0.0f);
            }
    };
    auto hand_v = [&](int c) {
        float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 y = make_float4(to_f32(vn[j][0]), to_f32(vn[j][1]), to_f32(vn[j][2]), to_f32(vn[j][3]));
            m0 = fmaxf(m0, fmaxf(fabsf(y.x), fabsf(y.y)));
            m1 = fmaxf(m1, fmaxf(fabsf(y.z), fabsf(y.w)));
            xb[c & 1].v[j][lane] = y;
        }
        xb[c & 1].v_max[lane] = make_float2(quad_max(m0), quad_max(m1));
    };
    auto product = [&](int c, float (&sq)[4][4]) {  // S Q^T
        const uint32_t qs = sm100::smem_u32(smem) + c % NS * SB + KT * 64 * DK;
        const X& x = xb[c & 1];
        const float2 inv = x.s_inv[lane];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int y = 0; y < 4; ++y) sq[j][y] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            const uint4 h4 = x.s[0][kk][lane], l4 = x.s[PREC ? 1 : 0][kk][lane];
            const uint32_t hi[4] = {h4.x, h4.y, h4.z, h4.w}, lo[4] = {l4.x, l4.y, l4.z, l4.w};
            uint32_t b[2][KT][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < KT; ++t) ldsm4(b[h][t], addr_nk<DK>(qs + t * 64 * DK, 2 * h, kk, lane));
#pragma unroll
            for (int h = 0; h < 2; ++h) { mma(sq[2 * h], hi, b[h][0][0], b[h][0][1]); mma(sq[2 * h + 1], hi, b[h][0][2], b[h][0][3]); }
            if (PREC)
#pragma unroll
                for (int h = 0; h < 2; ++h) { mma(sq[2 * h], lo, b[h][0][0], b[h][0][1]); mma(sq[2 * h + 1], lo, b[h][0][2], b[h][0][3]); }
            if (KT == 2)
#pragma unroll
                for (int h = 0; h < 2; ++h) { mma(sq[2 * h], hi, b[h][KT - 1][0], b[h][KT - 1][1]); mma(sq[2 * h + 1], hi, b[h][KT - 1][2], b[h][KT - 1][3]); }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) { sq[j][0] *= inv.x; sq[j][1] *= inv.x; sq[j][2] *= inv.y; sq[j][3] *= inv.y; }
    };
    auto finish = [&](int c, const float (&sq)[4][4]) {  // O = b S Q^T + u A^T
        const uint32_t as = sm100::smem_u32(smem) + c % NS * SB + 2 * KT * 64 * DK + 4096;
        const float* sc = reinterpret_cast<const float*>(smem + c % NS * SB + 2 * KT * 64 * DK + 8192);
        const X& x = xb[c & 1];
        float in[4][4] = {};
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint4 h4 = x.u[0][kk][lane], l4 = x.u[PREC ? 1 : 0][kk][lane];
            const uint32_t hi[4] = {h4.x, h4.y, h4.z, h4.w}, lo[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
            for (int h = kk; h < 2; ++h) {
                uint32_t bh[4], bl[4];
                ldsm4(bh, addr_nk<32>(as, 2 * h, kk, lane));
                mma(in[2 * h], hi, bh[0], bh[1]); mma(in[2 * h + 1], hi, bh[2], bh[3]);
                if (PREC) {
                    ldsm4(bl, addr_nk<32>(as + 2048, 2 * h, kk, lane));
                    mma(in[2 * h], lo, bh[0], bh[1]); mma(in[2 * h + 1], lo, bh[2], bh[3]);
                    mma(in[2 * h], hi, bl[0], bl[1]); mma(in[2 * h + 1], hi, bl[2], bl[3]);
                }
            }
        }
        const float2 inv = x.u_inv[lane];
        const float ainv = sc[kRecHead * 32 + kHeadA], q0 = inv.x * ainv, q1 = inv.y * ainv;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 bq = *reinterpret_cast<const float2*>(sc + kRecBq * 32 + j * 8 + 2 * c4);
            in[j][0] = fmaf(sq[j][0], bq.x, in[j][0] * q0); in[j][1] = fmaf(sq[j][1], bq.y, in[j][1] * q0);
            in[j][2] = fmaf(sq[j][2], bq.x, in[j][2] * q1); in[j][3] = fmaf(sq[j][3], bq.y, in[j][3] * q1);
        }
        if (a.save) {
            float* dst = reinterpret_cast<float*>(a.ws + a.l.o) + ((size_t)n * nch + c) * a.l.dvp * kDeltaChunk;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                *reinterpret_cast<float2*>(dst + r0 * kDeltaChunk + j * 8 + 2 * c4) = make_float2(in[j][0], in[j][1]);
                *reinterpret_cast<float2*>(dst + r1 * kDeltaChunk + j * 8 + 2 * c4) = make_float2(in[j][2], in[j][3]);
            }
        }
        if (o) {
            IO* p = o + ((size_t)c * kDeltaChunk + 2 * c4) * s.dv + r0;
            const int left = s.L - c * kDeltaChunk - 2 * c4;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int t = j * 8 + (y & 1);
                    if (t < left && (y < 2 ? ok0 : ok1)) p[(size_t)t * s.dv + (y < 2 ? 0 : 8)] = from_f32<IO>(in[j][y]);
                }
        }
    };
    load_v(0);
    hand_v(0);
    __syncthreads();
    if (nch > 1) load_v(1);
    float sq[4][4];
    for (int i = 0; i <= nch; ++i) {
        if (active && i > 0) finish(i - 1, sq);
        if (i < nch) {
            sm100::mbar_wait(&full[i % NS], (i / NS) & 1, wait, 903);
            if (active) product(i, sq);
        }
        if (i + 1 < nch) hand_v(i + 1);  // the chain reads chunk i's now
        if (i + 2 < nch) load_v(i + 2);
        if (i < nch) __syncthreads();    // chunk i is through the chain, chunk i - 1 through here
        if (fetches && i > 0 && i - 1 + NS < nch) fetch(i - 1 + NS);
        __syncwarp();
    }
}

template <typename IO, int DK, int KT, bool PREC> int launch(const DeltaArgs& a, cudaStream_t st) {
    auto kernel = delta_fwd_kernel<IO, DK, KT, PREC>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, fwd_smem<DK, KT, PREC>(4));
    if (e != cudaSuccess) return (int)e;
    // slices per CTA: they share the tiles in shared memory, but a chain with a scheduler of its own walks fastest
    int w = 4;
    while (w > 1 && a.l.N * ((a.l.slices + w - 1) / w) < 96) w >>= 1;
    const unsigned grid = (unsigned)(a.l.N * ((a.l.slices + w - 1) / w));
    kernel<<<grid, 2 * w * 32, fwd_smem<DK, KT, PREC>(w), st>>>(a, w);
    return (int)cudaGetLastError();
}

}  // namespace

int delta_fwd_launch(const DeltaArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.s.f32) return a.l.DK == 64 ? launch<float, 64, 2, true>(a, st) : launch<float, 128, 2, true>(a, st);
    if (a.save) return a.l.DK == 64 ? launch<__nv_bfloat16, 64, 1, true>(a, st) : launch<__nv_bfloat16, 128, 1, true>(a, st);
    return a.l.DK == 64 ? launch<__nv_bfloat16, 64, 1, false>(a, st) : launch<__nv_bfloat16, 128, 1, false>(a, st);
}

}  // namespace e2ttt
