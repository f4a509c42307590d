// Gated linear recurrence, reverse pass.  The adjoint of h runs backwards by the same rule: lam_t = d_h_t + a_{t+1} lam_{t+1}.  A CTA has 64 channels of a sequence and goes
// through its tiles of 64 tokens from the last to the first; a lane has two channels, a warp eight tokens.  A tile starts from its saved state and from the adjoint that the
// tokens after it hand on.  Per run of tokens P (the product of the a_t), the end h' of the states from zero and the adjoint v' handed on from zero meet in shared memory, once
// for both directions; where the tiles of a sequence are dealt out to a cluster's CTAs, P and v' of a tile meet through distributed shared memory, as in the forward.
// With a, i, s the gates and u = i x:
//   d_x = lam s i,   d_a_in = lam s u (1 - i),   d_log_a = a lam (h_{t-1} - a u / s),   d_a_decay = d_log_a log_a (1 - sg),   d_rate = -sum d_log_a sg.
#include <type_traits>

#include "api_checks.h"
#include "pack8.cuh"
#include "scan_common.cuh"

namespace e2ttt {
namespace {
using namespace scan;

constexpr int kTok = 8, kTile = kTok * kWarps, kStages = 2;
static_assert(kTile == kScanSpan, "a tile starts from a saved state");

struct Meet {
    float4 runs[2][kWarps][32];  // P and h' of a warp's tokens
    float4 parts[2][8][32];      // P and v' of a CTA's tile
    float2 ends[2][kWarps][32];  // v' of a warp's tokens
};

// what a warp has under way of a tile
template <typename IO, int NT, bool PACK> struct Rows {
    IO in[NT][kTok][kScanCh];
    IO d_h[kTok][kScanCh];
};
template <typename IO, int NT> struct Rows<IO, NT, true> {
    uint8_t codes[NT][kTok][kScanCh];
    IO d_h[kTok][kScanCh];
    uint8_t scales[NT][kTok][2];
};

template <int K, typename IO, int NT> __device__ __forceinline__ float2 input(const Rows<IO, NT, false>& r, int j, int lane) { return row2<IO>(r.in[K][j], lane); }
template <int K, typename IO, int NT> __device__ __forceinline__ float2 input(const Rows<IO, NT, true>& r, int j, int lane) {
    const uint32_t w = reinterpret_cast<const uint16_t*>(r.codes[K][j])[lane];
    return mul2(make_float2(pack8::number<0>(w), pack8::number<1>(w)), dup(pack8::scale(r.scales[K][j][lane >> 4])));
}

template <typename IO, bool GATE, bool UNIT, bool PACK>
__global__ void __launch_bounds__(kThreads, sizeof(IO) == 2 ? 2 : 1) scan_bwd_kernel(const ScanBwdArgs ba, const int by, const bool pair, const int parts) {
    constexpr int NT = GATE ? 3 : 2;
    using R = Rows<IO, NT, PACK>;
    extern __shared__ __align__(16) char smem[];
    Meet& meet = *reinterpret_cast<Meet*>(smem);
    const ScanArgs& a = ba.f;
    const int D = a.s.D, L = a.s.L, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    R* ring = reinterpret_cast<R*>(smem + sizeof(Meet)) + warp * kStages;
    const int64_t blocks = a.s.blocks(), tiles = a.s.spans(), unit = blockIdx.x / parts, b = unit / blocks;
    const int part = blockIdx.x - (int)(unit * parts), first = (int)(unit - b * blocks) * kScanCh;
    const int c0 = first + 2 * lane, n = max(0, min(2, D - c0));
    const int64_t seq = b * L * (int64_t)D;
    float2 rate = load2<float>(a.rate, c0, n, false);
    const bool near = __syncthreads_and(rate.x <= 0.25f && rate.y <= 0.25f);
    rate = make_float2(-rate.x, -rate.y);
    float2 carry = ba.dh_final ? load2<float>(ba.dh_final, b * D + c0, n, false) : dup(0.0f), sum = dup(0.0f);
    if (parts > 1) cluster_sync();  // the others' shared memory is there
    unsigned next_first = 0;
    auto load = [&](int64_t tile, int slot) {
        next_first = 0;
        if (tile >= 0 && tile < tiles) {
            const int t = (int)(tile * kTile) + warp * kTok;
            R& to = ring[slot];
            if constexpr (PACK) {
                const int64_t row = unit * tiles * kScanSpan + t;
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    copy16(&to.codes[k][0][0] + lane * 16, a.codes + k * a.code_step + row * kScanCh + lane * 16, true);
                    if (lane == k) copy16(&to.scales[k][0][0], a.scales + k * a.scale_step + row * 2, true);
                }
            } else {
                copy_rows<IO, kTok>(to.in[0][0], static_cast<const IO*>(a.x), seq, t, L, first, D, by, lane);
                copy_rows<IO, kTok>(to.in[1][0], static_cast<const IO*>(a.r), seq, t, L, first, D, by, lane);
                if constexpr (GATE) copy_rows<IO, kTok>(to.in[2][0], static_cast<const IO*>(a.g), seq, t, L, first, D, by, lane);
            }
            copy_rows<IO, kTok>(to.d_h[0], static_cast<const IO*>(ba.d_h), seq, t, L, first, D, by, lane);
            if (a.starts && lane < kTok && t + lane < L) next_first = a.starts[b * L + t + lane];
        }
        copy_commit();
    };
    const int64_t turns = (tiles + parts - 1) / parts;
    load((turns - 1) * parts + part, 0);
    unsigned byte0 = next_first;
    load((turns - 2) * parts + part, 1);
    int slot = 0;
    for (int64_t turn = turns - 1; turn >= 0; --turn, slot ^= 1) {
        const int64_t tile = turn * parts + part;
        const int t0 = (int)min(tile * kTile + warp * kTok, (int64_t)L), have = min(kTok, L - t0);
        const unsigned starts = __ballot_sync(kAll, byte0 != 0);
        byte0 = next_first;
        float2 state = tile < tiles ? load2<float>(a.states, (b * tiles + tile) * D + c0, n, false) : dup(0.0f);
        const R& rows = ring[slot];
        copy_wait<kStages - 1>();
        __syncwarp();
        float2 c[kTok], wr[kTok], wi[kTok], rs[kTok];
        unsigned far = 0;  // two bits a token
        float2 hh = dup(0.0f), pp = dup(1.0f), v = dup(0.0f);
        const bool plain = near && have == kTok && !starts;  // all tokens are there, none is a start, no decay is far from 1
        auto scale = [&](auto is_plain, int j) {             // s of token j
            constexpr bool PLAIN = decltype(is_plain)::value;
            if (!UNIT || (!PLAIN && (starts >> j & 1))) return dup(1.0f);
            float2 one = mul2(make_float2(-c[j].x, -c[j].y), add2(c[j], dup(2.0f)));
            if (!PLAIN && (far >> 2 * j & 1)) one.x = fmaf(-c[j].x, c[j].x, 1.0f);
            if (!PLAIN && (far >> 2 * j & 2)) one.y = fmaf(-c[j].y, c[j].y, 1.0f);
            return mul2(one, rs[j]);
        };
        auto gather = [&](auto is_plain) {
            constexpr bool PLAIN = decltype(is_plain)::value;
#pragma unroll
            for (int j = 0; j < kTok; ++j) {
                c[j] = wr[j] = wi[j] = rs[j] = dup(0.0f);
                if (!PLAIN && j >= have) continue;
                float2 u = input<0>(rows, j, lane);
                wr[j] = smaller_part2<IO>(input<1>(rows, j, lane));
                if constexpr (GATE) {
                    wi[j] = smaller_part2<IO>(input<2>(rows, j, lane));
                    u = mul2(u, open2(wi[j]));
                }
                const Decay d = decay<IO, UNIT, PLAIN>(open2(wr[j]), rate);
                c[j] = d.c;
                if (!PLAIN) far |= d.far << 2 * j;
                if (UNIT) rs[j] = inv_sqrt2<IO>(d.one);
                if (!PLAIN && (starts >> j & 1)) {
                    hh = u;
                    pp = dup(0.0f);
                    continue;
                }
                if (UNIT) u = mul2(u, mul2(d.one, rs[j]));
                hh = add2(fade<PLAIN>(hh, d.c, d.far), u);
                pp = fade<PLAIN>(pp, d.c, d.far);
            }
#pragma unroll
            for (int j = kTok - 1; j >= 0; --j) {
                if (!PLAIN && j >= have) continue;
                v = add2(v, row2<IO>(rows.d_h[j], lane));
                v = !PLAIN && (starts >> j & 1) ? dup(0.0f) : fade<PLAIN>(v, c[j], far >> 2 * j);
            }
        };
        if (plain) gather(std::true_type{});
        else gather(std::false_type{});
        meet.runs[slot][warp][lane] = make_float4(pp.x, pp.y, hh.x, hh.y);
        meet.ends[slot][warp][lane] = v;
        __syncthreads();
        float2 P_in = dup(1.0f), own = parts == 1 ? carry : dup(0.0f), P_all = P_in, all = own;  // the warps after this one; all of them
#pragma unroll
        for (int w = kWarps - 1; w >= 0; --w) {
            const float4 q = meet.runs[slot][w][lane];
            if (w == warp) {
                P_in = P_all;
                own = all;
            }
            if (w < warp) continue;
            all = through2(make_float2(q.x, q.y), all, meet.ends[slot][w][lane]);
            P_all = mul2(P_all, make_float2(q.x, q.y));
        }
        for (int w = warp - 1; w >= 0; --w) {
            const float4 q = meet.runs[slot][w][lane];
            all = through2(make_float2(q.x, q.y), all, meet.ends[slot][w][lane]);
            P_all = mul2(P_all, make_float2(q.x, q.y));
        }
        for (int w = 0; w < warp; ++w) {
            const float4 q = meet.runs[slot][w][lane];
            state = through2(make_float2(q.x, q.y), state, make_float2(q.z, q.w));
        }
        float2 in = own;
        if (parts == 1) {
            carry = all;
        } else {
            if (warp < parts) put_remote(&meet.parts[slot][part][lane], warp, make_float4(P_all.x, P_all.y, all.x, all.y));
            cluster_sync();
            for (int k = parts - 1; k >= 0; --k) {
                const float4 q = meet.parts[slot][k][lane];
                if (k == part) in = through2(P_in, carry, own);
                carry = through2(make_float2(q.x, q.y), carry, make_float2(q.z, q.w));
            }
        }
        auto spread = [&](auto is_plain) {
            constexpr bool PLAIN = decltype(is_plain)::value;
            float2 hp[kTok];  // the state before a token
#pragma unroll
            for (int j = 0; j < kTok; ++j) {
                hp[j] = state;
                if (!PLAIN && j >= have) continue;
                float2 u = input<0>(rows, j, lane);
                if (GATE) u = mul2(u, open2(wi[j]));
                if (!PLAIN && (starts >> j & 1)) state = u;
                else state = add2(fade<PLAIN>(state, c[j], far >> 2 * j), mul2(u, scale(is_plain, j)));
            }
            const int64_t at = seq + (int64_t)t0 * D + c0;
#pragma unroll
            for (int j = kTok - 1; j >= 0; --j) {
                if (!PLAIN && j >= have) continue;
                const bool start = !PLAIN && (starts >> j & 1);
                in = add2(in, row2<IO>(rows.d_h[j], lane));
                const float2 ls = mul2(in, scale(is_plain, j)), oi = open2(wi[j]);
                float2 u = input<0>(rows, j, lane);
                if (GATE) u = mul2(u, oi);
                store2<IO>(ba.d_x, at + (int64_t)j * D, n, pair, GATE ? mul2(ls, oi) : ls);
                if (GATE) store2<IO>(ba.d_g, at + (int64_t)j * D, n, pair, mul2(mul2(ls, u), closed2(wi[j])));
                in = start ? dup(0.0f) : fade<PLAIN>(in, c[j], far >> 2 * j);  // a lam
                float2 dl = dup(0.0f);                                        // d_log_a sg
                const float2 sg = open2(wr[j]);
                if (!start) {
                    float2 to = hp[j];
                    if (UNIT) {
                        const float2 ur = mul2(u, rs[j]), au = fade<PLAIN>(ur, c[j], far >> 2 * j);
                        to = add2(to, make_float2(-au.x, -au.y));
                    }
                    dl = mul2(mul2(in, to), sg);
                    sum = add2(sum, make_float2(-dl.x, -dl.y));
                }
                store2<IO>(ba.d_r, at + (int64_t)j * D, n, pair, mul2(mul2(dl, rate), closed2(wr[j])));
            }
        };
        if (plain) spread(std::true_type{});
        else spread(std::false_type{});
        __syncwarp();
        load((turn - 2) * parts + part, slot);
    }
    if (part == 0 && warp == 0) store2<float>(ba.dh_init, b * D + c0, n, false, carry);
    __syncthreads();
    meet.ends[0][warp][lane] = sum;
    __syncthreads();
    copy_wait<0>();
    if (warp != 0) return;
    sum = meet.ends[0][0][lane];
    for (int w = 1; w < kWarps; ++w) sum = add2(sum, meet.ends[0][w][lane]);
    store2<float>(ba.part, (b * parts + part) * D + c0, n, false, sum);
}

// d_rate: the sums of all sequences and parts, in an order that depends on their number alone
__global__ void __launch_bounds__(256) scan_rate_kernel(const float* part, float* d_rate, const int64_t rows, const int D) {
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float y = 0.0f;
    if (c < D)
        for (int64_t i = warp; i < rows; i += 8) y += part[i * D + c];
    sums[warp][lane] = y;
    __syncthreads();
    if (warp != 0 || c >= D) return;
    for (int w = 1; w < 8; ++w) y += sums[w][lane];
    d_rate[c] = y;
}

template <typename IO, bool GATE, bool UNIT, bool PACK> int launch(const ScanBwdArgs& b, int by, bool pair, cudaStream_t st) {
    auto kernel = scan_bwd_kernel<IO, GATE, UNIT, PACK>;
    cudaError_t e = allow_shared_memory<scan_bwd_kernel<IO, GATE, UNIT, PACK>>();
    if (e != cudaSuccess) return (int)e;
    const ScanShape& s = b.f.s;
    const int parts = scan_bwd_parts(s);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.B * s.blocks() * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Meet) + kStages * kWarps * sizeof(Rows<IO, GATE ? 3 : 2, PACK>);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kernel, b, by, pair, parts);
    if (e != cudaSuccess) return (int)e;
    scan_rate_kernel<<<(s.D + 31) / 32, 256, 0, st>>>(b.part, b.d_rate, (int64_t)s.B * parts, s.D);
    return (int)cudaGetLastError();
}
template <typename IO, bool GATE, bool UNIT> int launch(const ScanBwdArgs& b, int by, bool pair, cudaStream_t st) {
    return b.f.codes ? launch<IO, GATE, UNIT, true>(b, by, pair, st) : launch<IO, GATE, UNIT, false>(b, by, pair, st);
}
template <typename IO> int dispatch(const ScanBwdArgs& b, int by, bool pair, cudaStream_t st) {
    if (b.f.s.gate) return b.f.s.unit ? launch<IO, true, true>(b, by, pair, st) : launch<IO, true, false>(b, by, pair, st);
    return b.f.s.unit ? launch<IO, false, true>(b, by, pair, st) : launch<IO, false, false>(b, by, pair, st);
}

}  // namespace

int scan_bwd_parts(const ScanShape& s) {
    const int64_t units = s.B * s.blocks();
    int parts = 1;
    while (parts < 8 && units * parts < 296 && parts < s.spans()) parts *= 2;
    return parts;
}

int scan_bwd_launch(const ScanBwdArgs& b, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    uintptr_t in = reinterpret_cast<uintptr_t>(b.d_h), out = 0;
    if (!b.f.codes) in |= reinterpret_cast<uintptr_t>(b.f.x) | reinterpret_cast<uintptr_t>(b.f.r) | reinterpret_cast<uintptr_t>(b.f.g);
    for (const void* p : {b.d_x, b.d_r, b.d_g}) out |= reinterpret_cast<uintptr_t>(p);
    const int by = reads_by(b.f.s.D, b.f.s.f32, in);
    const bool pair = b.f.s.D % 2 == 0 && out % (b.f.s.f32 ? 8 : 4) == 0;
    return b.f.s.f32 ? dispatch<float>(b, by, pair, st) : dispatch<__nv_bfloat16>(b, by, pair, st);
}

}  // namespace e2ttt
