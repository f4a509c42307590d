// Gated delta rule, what does not depend on the state: one warp per chunk of 32 tokens and query / key head.
// It writes the chunk's queries and keys as fp16 tiles (scaled by powers of two, zero-padded, swizzled: the kernels that walk the chunks fetch
// them with bulk copies whatever the caller's width and alignment), and for every value head of the group the record of delta.h:
// T, A and the products of the decays.  All chunks run side by side.
// Bound by what it issues and by the latency of a chunk's dependent steps, with 12 chunks at a time on an SM, before memory: 64 heads of 4096 tokens,
// 128 wide, bf16, each with its own queries and keys, in 92 us (344 MB: 53 us at 6.5 TB/s); 64 value heads on 16 of those with what the reverse
// pass needs in 97 us (260 MB), each warp with four value heads one after the other.
#include "api_checks.h"
#include "delta_common.cuh"

namespace e2ttt {
namespace {
using namespace delta;

constexpr int kWarps = 4;

// the tiles, and over them, once their products are in registers, N (32 rows of 36) and its inverse (32 rows of 33); then the tokens' scalars
constexpr int kTriangles = 4608 + 4224;
template <int DK, int KT> constexpr int prep_work_bytes() { return 2 * KT * 64 * DK > kTriangles ? 2 * KT * 64 * DK : kTriangles; }
template <int DK, int KT> constexpr int prep_warp_bytes() { return prep_work_bytes<DK, KT>() + 256 + 256; }

// largest magnitude of a row tile, then its scaled terms to shared memory and to the workspace; norm: the 2-norm of the whole tile
template <typename IO, int DK, int KT>
__device__ __forceinline__ float stage_rows(const IO* src, int rows, int d, bool vec, char* sm, char* out, int lane, float& norm) {
    constexpr int P = DK / 8;  // 16-byte pieces of a tile row
    float m = 0.0f;
    auto load = [&](int i, float (&x)[8]) {
        const int r = i / P, c = (i % P) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.0f;
        if (r >= rows || c >= d) return;
        const IO* p = src + (size_t)r * d + c;
        if (vec) {
            if (sizeof(IO) == 2) {
                const uint4 raw = *reinterpret_cast<const uint4*>(p);
                const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[2 * j] = __uint_as_float(w[j] << 16);
                    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                }
            } else {
                const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
                x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < d) x[j] = to_f32(p[j]);
        }
    };
    float sq0 = 0.0f, sq1 = 0.0f;  // squares, scaled
    auto put = [&](int i, float (&x)[8], float s) {
        uint4 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            mul2(x[j], x[j + 1], x[j], x[j + 1], s, s);
            fma2(sq0, sq1, x[j], x[j + 1], x[j], x[j + 1], sq0, sq1);
        }
        split(x[0], x[1], hi.x, lo.x);
        split(x[2], x[3], hi.y, lo.y);
        split(x[4], x[5], hi.z, lo.z);
        split(x[6], x[7], hi.w, lo.w);
        const uint32_t at = tile_at<DK>(i / P, i % P);
        *reinterpret_cast<uint4*>(sm + at) = hi;
        *reinterpret_cast<uint4*>(out + at) = hi;
        if (KT == 2) {
            *reinterpret_cast<uint4*>(sm + 64 * DK + at) = lo;
            *reinterpret_cast<uint4*>(out + 64 * DK + at) = lo;
        }
    };
    float s, inv;
    if (sizeof(IO) == 2 && vec) {  // the whole tile in flight: 16 bytes a lane and load, one round trip
        uint4 raw[P];
        const bool full = rows == kDeltaChunk && d == DK;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int r = (i * 32 + lane) / P, c = (i * 32 + lane) % P * 8;
            raw[i] = full || (r < rows && c < d) ? *reinterpret_cast<const uint4*>(src + (size_t)r * d + c) : make_uint4(0, 0, 0, 0);
        }
        uint32_t top = 0;  // largest magnitude on the bits: both halves of a word at a time
#pragma unroll
        for (int i = 0; i < P; ++i) {
            top = __vmaxu2(top, raw[i].x & 0x7fff7fffu);
            top = __vmaxu2(top, raw[i].y & 0x7fff7fffu);
            top = __vmaxu2(top, raw[i].z & 0x7fff7fffu);
            top = __vmaxu2(top, raw[i].w & 0x7fff7fffu);
        }
        m = __uint_as_float(max(top << 16, top & 0xffff0000u));
        if (!(m <= 3.4e38f)) m = __uint_as_float(0x7f000000u);  // infinities and NaNs: any scale
        pow2_scale(warp_max(m), s, inv);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
            float x[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
            put(i * 32 + lane, x, s);
        }
        norm = sqrtf(warp_sum(sq0 + sq1)) * inv;
        return inv;
    }
#pragma unroll 4
    for (int i = lane; i < 32 * P; i += 32) {
        float x[8];
        load(i, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(x[j]));
    }
    pow2_scale(warp_max(m), s, inv);
#pragma unroll 4
    for (int i = lane; i < 32 * P; i += 32) {
        float x[8];
        load(i, x);  // from L1
        put(i, x, s);
    }
    norm = sqrtf(warp_sum(sq0 + sq1)) * inv;
    return inv;
}

// rows x keys on and below the diagonal blocks: tiles (m, n) with n <= 2 m + 1
template <int DK, int KT> __device__ __forceinline__ void gram(uint32_t rows, uint32_t keys, float (&c)[6][4], int lane) {
#pragma unroll
    for (int i = 0; i < 6; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.0f;
#pragma unroll 2
    for (int kk = 0; kk < DK / 16; ++kk) {
        uint32_t a0[KT][4], a1[KT][4], b0[KT][4], b1[KT][4];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            ldsm4(a0[t], addr_mk<DK>(rows + t * 64 * DK, 0, kk, lane));
            ldsm4(a1[t], addr_mk<DK>(rows + t * 64 * DK, 16, kk, lane));
            ldsm4(b0[t], addr_nk<DK>(keys + t * 64 * DK, 0, kk, lane));
            ldsm4(b1[t], addr_nk<DK>(keys + t * 64 * DK, 2, kk, lane));
        }
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int u = 0; u + t < KT; ++u) {
                mma(c[0], a0[t], b0[u][0], b0[u][1]);
                mma(c[1], a0[t], b0[u][2], b0[u][3]);
                mma(c[2], a1[t], b0[u][0], b0[u][1]);
                mma(c[3], a1[t], b0[u][2], b0[u][3]);
                mma(c[4], a1[t], b1[u][0], b1[u][1]);
                mma(c[5], a1[t], b1[u][2], b1[u][3]);
            }
    }
}

// (I + N)^-1 of a strictly lower N column by column, lane = column: x_t = [t == lane] - sum_{i < t} N_ti x_i, four rows at a time; the columns
// in shared memory (rows of 33).  Rolled: with all rows written out the warps of an SM, each at a place of its own, waited for instructions a
// third of their time.  Two terms to `out`, then by rows; the largest sums of magnitudes of a row and of a column.
__device__ __forceinline__ float invert(const float* Nm, float* xs, char* out, int lane, float& rows, float& cols) {
    float col = 0.0f;
#pragma unroll 1
    for (int t = 0; t < 32; t += 4) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = t + k == lane ? 1.0f : 0.0f;
#pragma unroll 2
        for (int i = 0; i < t; i += 4) {
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = xs[(i + k) * 33 + lane];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 w = *reinterpret_cast<const float4*>(Nm + (t + k) * 36 + i);
                y[k] = fmaf(-w.x, x[0], y[k]); y[k] = fmaf(-w.y, x[1], y[k]);
                y[k] = fmaf(-w.z, x[2], y[k]); y[k] = fmaf(-w.w, x[3], y[k]);
            }
        }
        const float* d = Nm + t * 36 + t;
        y[1] = fmaf(-d[36], y[0], y[1]);
        y[2] = fmaf(-d[72], y[0], y[2]); y[2] = fmaf(-d[73], y[1], y[2]);
        y[3] = fmaf(-d[108], y[0], y[3]); y[3] = fmaf(-d[109], y[1], y[3]); y[3] = fmaf(-d[110], y[2], y[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            xs[(t + k) * 33 + lane] = y[k];
            col += fabsf(y[k]);
        }
    }
    __syncwarp();
    const float* row = xs + lane * 33;  // lane = row
    float sum = 0.0f, most = 0.0f;
#pragma unroll 8
    for (int i = 0; i < 32; ++i) {
        const float x = fabsf(row[i]);
        sum += x;
        most = fmaxf(most, x);
    }
    rows = warp_max(sum);
    cols = warp_max(col);
    float s, inv;
    pow2_scale(warp_max(most), s, inv);
#pragma unroll 1
    for (int piece = 0; piece < 4; ++piece) {
        uint4 hi, lo;
        const float* x = row + piece * 8;
        split(x[0] * s, x[1] * s, hi.x, lo.x);
        split(x[2] * s, x[3] * s, hi.y, lo.y);
        split(x[4] * s, x[5] * s, hi.z, lo.z);
        split(x[6] * s, x[7] * s, hi.w, lo.w);
        const uint32_t at = tile_at<32>(lane, piece);
        *reinterpret_cast<uint4*>(out + at) = hi;
        *reinterpret_cast<uint4*>(out + 2048 + at) = lo;
    }
    __syncwarp();
    return inv;
}

template <typename IO, int DK, int KT>
__global__ void __launch_bounds__(kWarps * 32, 3) delta_prep_kernel(const DeltaArgs a, const bool vec) {
    extern __shared__ __align__(1024) char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const DeltaShape& s = a.s;
    const int64_t item = (int64_t)blockIdx.x * kWarps + warp;
    if (item >= a.l.Nk * a.l.nch) return;
    if (item == 0 && lane == 0) *reinterpret_cast<int*>(a.ws) = 0;  // the status word
    const int64_t nk = item / a.l.nch;
    const int c = (int)(item % a.l.nch);
    const int t0 = c * kDeltaChunk, rows = min(kDeltaChunk, s.L - t0);
    char* sm = smem + warp * prep_warp_bytes<DK, KT>();
    float* Nm = reinterpret_cast<float*>(sm);
    float* xs = reinterpret_cast<float*>(sm + 4608);
    double* run = reinterpret_cast<double*>(sm + prep_work_bytes<DK, KT>());
    float* eta_s = reinterpret_cast<float*>(run + 32);
    float* norm_s = eta_s + 32;  // |k|^2, in units of the tile
    char* out = a.ws + a.l.qk + (size_t)item * a.l.qk_bytes;
    const size_t row0 = ((size_t)nk * s.L + t0) * s.dk;
    float ik = 1.0f, iq = 1.0f, q_norm = 0.0f;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        ik = iq;
        iq = stage_rows<IO, DK, KT>(reinterpret_cast<const IO*>(which ? a.q : a.k) + row0, rows, s.dk, vec, sm + which * KT * 64 * DK,
                                    out + which * KT * 64 * DK, lane, q_norm);
    }
    __syncwarp();
    const uint32_t ks = sm100::smem_u32(sm), qs = ks + KT * 64 * DK;
    float kk[6][4], qk[6][4];
    gram<DK, KT>(ks, ks, kk, lane);
    gram<DK, KT>(qs, ks, qk, lane);
    __syncwarp();
    const int g = lane >> 2, c4 = lane & 3, r = s.H / s.Hk;
#pragma unroll
    for (int i = 0; i < 6; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int t = (i < 2 ? 0 : 16) + g + (x >> 1) * 8, u = (i < 2 ? i * 8 : (i - 2) * 8) + 2 * c4 + (x & 1);
            if (u == t) norm_s[t] = kk[i][x];
        }
    __syncwarp();
    const float kn = sqrtf(norm_s[lane]) * ik;
    const float ik_t = norm_s[lane] == 0.0f ? 0.0f : ik;  // a token without a key has factors of 0: no scale is stretched for it
    const int64_t b = nk / s.Hk, hk = nk % s.Hk;
    for (int j = 0; j < r; ++j) {
        const int64_t n = b * s.H + hk * r + j;
        const size_t gate = (size_t)n * s.L + t0;
        // gates: lane = token.  The decays' logarithms are summed in 64 bits (the differences of long sums are what counts); below -1000
        // a decay is 0 in 32 bits all the same, and infinities leave the differences.
        float lg = lane < rows ? a.log_gamma[gate + lane] : 0.0f;
        const float eta = lane < rows ? a.eta[gate + lane] : 0.0f;
        if (lg < -1000.0f) lg = -1000.0f;
        double sum = (double)lg;
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            const double y = __shfl_up_sync(kAll, sum, i);
            if (lane >= i) sum += y;
        }
        const double end = __shfl_sync(kAll, sum, 31);
        __syncwarp();
        run[lane] = sum;
        eta_s[lane] = eta;
        __syncwarp();
        char* rec = a.ws + a.l.rec + ((size_t)n * a.l.nch + c) * a.l.rec_bytes;
        float* sc = reinterpret_cast<float*>(rec + 8192);
        const float bt = expf((float)sum), dend = expf((float)(end - sum));
        sc[kRecBk * 32 + lane] = bt * ik_t;
        sc[kRecBq * 32 + lane] = bt * iq * s.scale;
        sc[kRecEta * 32 + lane] = eta;
        sc[kRecDend * 32 + lane] = dend * ik_t;
        sc[kRecW * 32 + lane] = eta * dend * ik_t;
        sc[kRecZ * 32 + lane] = eta * bt * ik_t;
        // N = strict(D (k k^T)) eta to shared memory, A = lower(D (q k^T)) scale to the record
        float amax = 0.0f, emax = 0.0f, av[6][4], gk[6][4];  // gk: strict(D (k k^T))
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            const int m0 = i < 2 ? 0 : 16, n0 = i < 2 ? i * 8 : (i - 2) * 8;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int t = m0 + g + (x >> 1) * 8, u = n0 + 2 * c4 + (x & 1);
                const float D = u <= t ? expf((float)(run[t] - run[u])) : 0.0f;
                gk[i][x] = u < t ? D * kk[i][x] * (ik * ik) : 0.0f;
                Nm[t * 36 + u] = gk[i][x] * eta_s[u];
                av[i][x] = u <= t ? D * qk[i][x] * (iq * ik * s.scale) : 0.0f;
                amax = fmaxf(amax, fabsf(av[i][x]));
                emax = fmaxf(emax, fabsf(av[i][x] * eta_s[u]));
            }
        }
        float as, ai, es, ei;
        pow2_scale(warp_max(amax), as, ai);
        pow2_scale(warp_max(emax), es, ei);
#pragma unroll
        for (int i = 0; i < 6; ++i) {  // the block above the diagonal is read by no product
            const int m0 = i < 2 ? 0 : 16, n0 = i < 2 ? i : i - 2;
            const float e0 = eta_s[n0 * 8 + 2 * c4], e1 = eta_s[n0 * 8 + 2 * c4 + 1];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint32_t hi, lo;
                const uint32_t at = tile_at<32>(m0 + g + x * 8, n0) + c4 * 4;
                split(av[i][2 * x] * e0 * es, av[i][2 * x + 1] * e1 * es, hi, lo);
                *reinterpret_cast<uint32_t*>(rec + 4096 + at) = hi;
                *reinterpret_cast<uint32_t*>(rec + 6144 + at) = lo;
                if (a.save) {
                    split(av[i][2 * x] * as, av[i][2 * x + 1] * as, hi, lo);
                    *reinterpret_cast<uint32_t*>(rec + 9216 + at) = hi;
                    *reinterpret_cast<uint32_t*>(rec + 11264 + at) = lo;
                }
            }
        }
        if (a.save) {
            float4* pairs = reinterpret_cast<float4*>(rec + kDeltaRecPairs);
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                pairs[i * 32 + lane] = make_float4(av[i][0], av[i][1], av[i][2], av[i][3]);
                pairs[(6 + i) * 32 + lane] = make_float4(gk[i][0], gk[i][1], gk[i][2], gk[i][3]);
            }
        }
        __syncwarp();
        // T, and with saved states the same with eta on the rows: what the reverse pass multiplies with
        float tsum = 0.0f, ti = 0.0f, ri = 0.0f, rsum, csum;
#pragma unroll 1
        for (int pass = 0; pass <= a.save; ++pass) {
            const float y = invert(Nm, xs, rec + (pass ? 13312 : 0), lane, rsum, csum);
            if (pass) { ri = y; break; }
            ti = y;
            tsum = rsum;
            if (!a.save) break;
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                const int m0 = i < 2 ? 0 : 16, n0 = i < 2 ? i * 8 : (i - 2) * 8;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int t = m0 + g + (x >> 1) * 8, u = n0 + 2 * c4 + (x & 1);
                    Nm[t * 36 + u] = gk[i][x] * eta_s[t];
                }
            }
            __syncwarp();
        }
        const float b_kn = warp_max(bt * kn), wmax = warp_max(fabsf(eta) * dend * ik_t), wsum = warp_sum(fabsf(eta) * dend * kn);
        const float ke = warp_max(dend * kn), zmax = warp_max(fabsf(eta) * bt * ik_t), zsum = warp_sum(fabsf(eta) * bt * kn);
        const float up = bt * 0x1p60f;  // squares of decays down to 2^-120 stay in range
        const float qsum = fabsf(s.scale) * (sqrtf(warp_sum(up * up)) * 0x1p-60f) * q_norm;
        if (lane == 0) {
            float* head = sc + kRecHead * 32;
            head[kHeadEnd] = expf((float)end);
            head[kHeadT] = ti;
            head[kHeadA] = ei;
            head[kHeadK] = ik;
            head[kHeadQ] = iq;
            head[kHeadR] = ri;
            head[kHeadKn] = b_kn;
            head[kHeadTsum] = tsum;
            head[kHeadAr] = ai;
            head[kHeadWmax] = wmax;
            head[kHeadWsum] = wsum;
            head[kHeadKe] = ke;
            head[kHeadRsum] = csum;
            head[kHeadZmax] = zmax;
            head[kHeadZsum] = zsum;
            head[kHeadQsum] = qsum;
        }
        __syncwarp();
    }
}

template <typename IO, int DK, int KT> int launch(const DeltaArgs& a, cudaStream_t st) {
    constexpr int bytes = kWarps * prep_warp_bytes<DK, KT>();
    auto kernel = delta_prep_kernel<IO, DK, KT>;
    cudaError_t e = allow_shared_memory<delta_prep_kernel<IO, DK, KT>>();
    if (e != cudaSuccess) return (int)e;
    const bool vec = a.s.dk % 8 == 0 && (reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k)) % 16 == 0;
    const unsigned grid = (unsigned)((a.l.Nk * a.l.nch + kWarps - 1) / kWarps);
    kernel<<<grid, kWarps * 32, bytes, st>>>(a, vec);
    return (int)cudaGetLastError();
}

}  // namespace

int delta_prep_launch(const DeltaArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.s.f32) return a.l.DK == 64 ? launch<float, 64, 2>(a, st) : launch<float, 128, 2>(a, st);
    return a.l.DK == 64 ? launch<__nv_bfloat16, 64, 1>(a, st) : launch<__nv_bfloat16, 128, 1>(a, st);
}

}  // namespace e2ttt
