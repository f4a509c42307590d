// Gated linear recurrence, reverse pass.  The adjoint of h runs backwards by the same rule: lam_t = d_h_t + a_{t+1} lam_{t+1}.  A CTA has 64 channels of a sequence and goes
// through its tiles of 64 tokens from the last to the first; a lane has two channels, a warp eight tokens.  A tile starts from its saved state and from the adjoint that the
// tokens after it hand on.  Per run of tokens P (the product of the a_t), the end h' of the states from zero and the adjoint v' handed on from zero meet in shared memory, once
// for both directions; where the tiles of a sequence are dealt out to a cluster's CTAs, P and v' of a tile meet through distributed shared memory, as in the forward.
// With a, i, s the gates and u = i x:
//   d_x = lam s i,   d_a_in = lam s u (1 - i),   d_log_a = a lam (h_{t-1} - a u / s),   d_a_decay = d_log_a log_a (1 - sg),   d_rate = -sum d_log_a sg.
// What does not depend on lam is computed before the meeting and kept: c, -s i, sg a u / s, sg and a_decay's factor in registers, s u (1 - i) in shared memory.
// Gradients go out through the place of what they are the gradients of, by the copy engine: stores from the threads between the steps held up the loads (162 to 217 us, as
// the compiler laid them).  16384 tokens of 2048 in bf16: 133 us (470 MB, 3.5 TB/s), 193 with rates of up to 4;
// with inputs in 8 bits 150 us (373 MB: decoding costs more than the bytes save); fp32 267 us.  Rows that the copy engine cannot read: 347 us for 2046 channels, 412 for 2047.
// Registers allow two CTAs on an SM (fp32: one); issue takes 47 % of its slots, the dependent steps of eight tokens back and forth the rest.
#include <type_traits>

#include "api_checks.h"
#include "pack8.cuh"
#include "scan_common.cuh"
#include "scan_map.h"

namespace e2ttt {
namespace {
using namespace scan;

constexpr int kTok = 8, kTile = kTok * kWarps, kStages = 2;
static_assert(kTile == kScanSpan, "a tile starts from a saved state");

struct Meet {
    float4 runs[2][kWarps][32];        // P and h' of a warp's tokens
    float2 ends[2][kWarps][32];        // v' of a warp's tokens
    float2 carry[2][32];               // the adjoint that a turn's tokens hand on
    uint64_t full[kWarps][kStages];
    Meeting meeting;
    float2 stash[kWarps][kTok][32];    // a thread's own, for want of registers
};

constexpr int kMeet = (sizeof(Meet) + 127) / 128 * 128;

// what a warp has under way of a tile
template <typename IO, int NT, bool PACK> struct alignas(128) Rows {
    IO in[NT][kTok][kScanCh];
    IO d_h[kTok][kScanCh];
    static constexpr int kBytes = (NT + 1) * kTok * kScanCh * (int)sizeof(IO);
};
template <typename IO, int NT> struct alignas(128) Rows<IO, NT, true> {
    uint8_t codes[NT][kTok][kScanCh];
    IO d_h[kTok][kScanCh];
    alignas(128) uint8_t scales[NT][kTok][2];
    static constexpr int kBytes = NT * kTok * (kScanCh + 2) + kTok * kScanCh * (int)sizeof(IO);
};

// where a warp's gradients wait to be stored by the copy engine: in the place of what they are the gradients of, or, with packed inputs, in a place of their own
template <typename IO, int NT, bool PACK> struct Outs {
    IO g[PACK ? NT : 1][kTok][kScanCh];
};

template <int K, typename IO, int NT> __device__ __forceinline__ float2 input(const Rows<IO, NT, false>& r, int j, int lane) { return row2<IO>(r.in[K][j], lane); }
template <int K, typename IO, int NT> __device__ __forceinline__ float2 logit(const Rows<IO, NT, false>& r, int j, int lane) { return logit2<IO>(r.in[K][j], lane); }
template <int K, typename IO, int NT> __device__ __forceinline__ float2 input(const Rows<IO, NT, true>& r, int j, int lane) {
    const uint32_t w = reinterpret_cast<const uint16_t*>(r.codes[K][j])[lane];
    // a block that is not finite has codes of 0 and an infinite scale: NaN
    const float s = __uint_as_float((uint32_t)r.scales[K][j][lane >> 4] << 23);
    return mul2(add2(make_float2(pack8::biased<0>(w), pack8::biased<1>(w)), dup(-8388736.0f)), dup(s));
}
template <int K, typename IO, int NT> __device__ __forceinline__ float2 logit(const Rows<IO, NT, true>& r, int j, int lane) { return capped(input<K>(r, j, lane)); }

// TILE: rows are read by kByTile
template <typename IO, bool GATE, bool UNIT, bool PACK, bool TILE>
__global__ void __launch_bounds__(kThreads, sizeof(IO) == 2 ? 2 : 1) scan_bwd_kernel(const ScanBwdArgs ba, const __grid_constant__ ScanMaps maps, const int by, const bool pair, const int parts) {
    constexpr int NT = GATE ? 3 : 2;
    using R = Rows<IO, NT, PACK>;
    extern __shared__ __align__(128) char smem[];
    Meet& meet = *reinterpret_cast<Meet*>(smem);
    const ScanArgs& a = ba.f;
    const int D = a.s.D, L = a.s.L, lane = threadIdx.x & 31, warp = __shfl_sync(kAll, threadIdx.x >> 5, 0);
    using O = Outs<IO, NT, PACK>;
    R* ring = reinterpret_cast<R*>(smem + kMeet) + warp * kStages;
    O* outs = reinterpret_cast<O*>(smem + kMeet + kWarps * kStages * sizeof(R)) + warp;
    const int64_t blocks = a.s.blocks(), tiles = a.s.spans(), unit = blockIdx.x / parts, b = unit / blocks;
    const int part = blockIdx.x - (int)(unit * parts), first = (int)(unit - b * blocks) * kScanCh;
    const int c0 = first + 2 * lane, n = max(0, min(2, D - c0));
    const bool whole = first + kScanCh <= D;  // all channels are there
    const int64_t seq = b * L * (int64_t)D;
    const bool even = (D & 1) == 0;  // rows of states (in the workspace) are pairs
    const Pairs pairs = make_pairs();
    float2 rate = load2<float>(a.rate, c0, n, false);
    const bool near = __syncthreads_and(whole && near_rate(rate.x) && near_rate(rate.y));
    rate = make_float2(-rate.x, -rate.y);
    float2 end = ba.dh_final ? load2<float>(ba.dh_final, b * D + c0, n, false) : dup(0.0f), sum = dup(0.0f);  // end: what the last turn hands on, in one warp
    const int ender = parts == 1 ? 0 : kWarps - 1;
    if (warp == ender) meet.carry[1][lane] = end;
    uint64_t* full = meet.full[warp];
    if (TILE && lane == 0) {
        for (int i = 0; i < kStages; ++i) sm100::mbar_init(&full[i], 1);
        sm100::fence_mbar_init();
    }
    __syncwarp();
    if (parts > 1) meeting_init(meet.meeting);
    auto has_rows = [&](int64_t tile) { return tile >= 0 && tile * kTile + warp * kTok < L; };
    unsigned next_first = 0;
    bool met = true;  // no wait of this warp has given up
    auto load = [&](int64_t tile, int slot) {
        next_first = 0;
        if ((!TILE || met) && has_rows(tile)) {
            const int t = (int)(tile * kTile) + warp * kTok;
            R& to = ring[slot];
            const int64_t row = unit * tiles * kScanSpan + t;
            if constexpr (TILE) {
                if (lane == 0) {
                    sm100::mbar_expect_tx(&full[slot], R::kBytes);
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        if constexpr (PACK) {
                            bulk_load(to.codes[k][0], a.codes + k * a.code_step + row * kScanCh, kTok * kScanCh, &full[slot]);
                            bulk_load(to.scales[k][0], a.scales + k * a.scale_step + row * 2, kTok * 2, &full[slot]);
                        } else {
                            tile_load(to.in[k][0], &maps.in[k], first, t, (int)b, &full[slot]);
                        }
                    }
                    tile_load(to.d_h[0], &maps.in[3], first, t, (int)b, &full[slot]);
                }
            } else {
                if constexpr (PACK) {
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        copy16(&to.codes[k][0][0] + lane * 16, a.codes + k * a.code_step + row * kScanCh + lane * 16);
                        if (lane == k) copy16(&to.scales[k][0][0], a.scales + k * a.scale_step + row * 2);
                    }
                } else {
                    copy_rows<IO, kTok>(to.in[0][0], static_cast<const IO*>(a.x), seq, t, L, first, D, by, lane);
                    copy_rows<IO, kTok>(to.in[1][0], static_cast<const IO*>(a.r), seq, t, L, first, D, by, lane);
                    if constexpr (GATE) copy_rows<IO, kTok>(to.in[2][0], static_cast<const IO*>(a.g), seq, t, L, first, D, by, lane);
                }
                copy_rows<IO, kTok>(to.d_h[0], static_cast<const IO*>(ba.d_h), seq, t, L, first, D, by, lane);
            }
            if (a.starts && lane < kTok && t + lane < L) next_first = a.starts[b * L + t + lane];
        }
        if (!TILE) copy_commit();
    };
    const int64_t turns = (tiles + parts - 1) / parts;
    load((turns - 1) * parts + part, 0);
    unsigned byte0 = next_first;
    load((turns - 2) * parts + part, 1);
    auto state_of = [&](int64_t tile) { return tile >= 0 && tile < tiles ? load2<float>(a.states, (b * tiles + tile) * D + c0, n, even) : dup(0.0f); };
    float2 next_state = state_of((turns - 1) * parts + part);  // a turn ahead
    int slot = 0;
    uint32_t parity = 0, taken = 0;  // taken: which phase a stage's barrier is in (a warp may have no tokens in the first turn)
    auto give_up = [&](bool next) {  // next: the next turn's rows are under way
        met = false;
        if constexpr (TILE) {
            if (next) (void)await_on<false>(&full[slot ^ 1], taken >> (slot ^ 1) & 1, sm100::kWaitCycles);
            if (lane == 0) bulk_read_done();
            __syncwarp();
            fill(ring, kNans, kStages * sizeof(R));
            if constexpr (PACK)
                for (int i = 0; i < kStages; ++i) fill(ring[i].codes, 0, sizeof(ring[i].codes));
        }
    };
    for (int64_t turn = turns - 1; turn >= 0; --turn, slot ^= 1, parity ^= slot == 0) {
        const int64_t tile = turn * parts + part;
        const int t0 = (int)min(tile * kTile + warp * kTok, (int64_t)L), have = min(kTok, L - t0);
        const unsigned starts = __ballot_sync(kAll, byte0 != 0);
        byte0 = next_first;
        float2 state = next_state;
        next_state = state_of(tile - parts);
        R& rows = ring[slot];
        if constexpr (!TILE) {
            copy_wait<kStages - 1>();
        } else if (have > 0) {
            if (met && !await<false>(&full[slot], taken >> slot & 1, a.wait_cycles)) {
                (void)await_on<false>(&full[slot], taken >> slot & 1, sm100::kWaitCycles);
                give_up(turn == turns - 1 && has_rows(tile - parts));
            }
            taken ^= 1u << slot;
        }
        __syncwarp();
        // of token j: c as in the forward; to_x = -s i, what -lam is multiplied with in d_x (with a^2 - 1 at hand -s takes no special function); to_r, first sg a u / s, then
        // sg (h_{t-1} - a u / s); sg; to_a = d_a_decay / (d_log_a sg).  In the stash: -s u (1 - i), what -lam is multiplied with in d_a_in.
        float2 c[kTok], to_x[kTok], to_r[kTok], sg[kTok], to_a[kTok];
        unsigned far = 0;  // two bits a token
        float2 hh = dup(0.0f), pp = dup(1.0f), v = dup(0.0f);
        const bool plain = near && have == kTok && !starts;  // all tokens and channels are there, none is a start, no decay is far from 1
        auto gather = [&](auto is_plain) {
            constexpr bool PLAIN = decltype(is_plain)::value;
#pragma unroll
            for (int j = 0; j < kTok; ++j) {
                if (!PLAIN) c[j] = to_x[j] = to_r[j] = sg[j] = to_a[j] = dup(0.0f);
                if (!PLAIN && j >= have) continue;
                const float2 x = input<0>(rows, j, lane), er = exp_neg<IO>(pairs, logit<1>(rows, j, lane));
                float2 ig = dup(1.0f), shut = dup(0.0f);
                if constexpr (GATE) {
                    const float2 eg = exp_neg<IO>(pairs, logit<2>(rows, j, lane));
                    ig = reciprocal<IO>(add2(eg, pairs.one));
                    shut = mul2(eg, ig);
                }
                sg[j] = reciprocal<IO>(add2(er, pairs.one));
                to_a[j] = mul2(rate, mul2(er, sg[j]));
                const Decay d = decay<IO, UNIT, PLAIN>(pairs, sg[j], rate);
                c[j] = d.c;
                if (!PLAIN) far |= d.far << 2 * j;
                const bool start = !PLAIN && (starts >> j & 1);
                to_r[j] = dup(0.0f);
                if (UNIT && !start) {
                    const float2 rs = inv_sqrt_minus<PLAIN>(d.minus);
                    to_r[j] = mul2(sg[j], fade<PLAIN>(mul2(mul2(x, ig), rs), d.c, d.far));
                    to_x[j] = mul2(ig, mul2(d.minus, rs));
                } else {
                    to_x[j] = mul2(ig, pairs.minus_one);
                }
                const float2 bj = mul2(to_x[j], x);
                if (GATE) meet.stash[warp][j][lane] = mul2(bj, shut);
                hh = fma2(bj, pairs.minus_one, start ? dup(0.0f) : fade<PLAIN>(hh, d.c, d.far));
                pp = !PLAIN && cut_by(starts, j) ? dup(kCut) : fade<PLAIN>(pp, d.c, d.far);
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
        if (TILE && turn != turns - 1) {  // the last turn's gradients have left its stage by now
            if (lane == 0) bulk_read_done();
            __syncwarp();
            load((turn - 1) * parts + part, slot ^ 1);
            byte0 = next_first;
        }
        meet.runs[slot][warp][lane] = make_float4(pp.x, pp.y, hh.x, hh.y);
        meet.ends[slot][warp][lane] = v;
        __syncthreads();
        float2 in = meet.carry[slot ^ 1][lane];  // what the tokens after the turn's hand on
        auto meet_others = [&](auto is_cut) {
            constexpr bool CUT = decltype(is_cut)::value;
#pragma unroll
            for (int w = 0; w < kWarps - 1; ++w) {
                if (w >= warp) break;
                const float4 q = meet.runs[slot][w][lane];
                state = through<CUT>(make_float2(q.x, q.y), state, make_float2(q.z, q.w));
            }
            if (parts == 1) {
#pragma unroll
                for (int w = kWarps - 1; w > 0; --w) {
                    if (w <= warp) break;
                    const float4 q = meet.runs[slot][w][lane];
                    in = through<CUT>(make_float2(q.x, q.y), in, meet.ends[slot][w][lane]);
                }
                if (warp == ender) meet.carry[slot][lane] = end = through<CUT>(pp, in, v);
                return;
            }
            float2 P_in = dup(1.0f), own = dup(0.0f);  // the warps after this one
#pragma unroll
            for (int w = kWarps - 1; w > 0; --w) {
                if (w <= warp) break;
                const float4 q = meet.runs[slot][w][lane];
                own = through<CUT>(make_float2(q.x, q.y), own, meet.ends[slot][w][lane]);
                P_in = both<CUT>(P_in, make_float2(q.x, q.y));
            }
            if (warp == 0 && met) send_part(meet.meeting, slot, part, parts, lane, both<CUT>(P_in, pp), through<CUT>(pp, own, v));
            if (met && !await<true>(&meet.meeting.full[slot], parity, a.wait_cycles)) {
                (void)await_on<true>(&meet.meeting.full[slot], parity, kSendCycles);
                give_up(has_rows(tile - parts));
            }
            for (int k = parts - 1; k > part; --k) {
                const float4 q = meet.meeting.parts[slot][k][lane];
                in = through<CUT>(make_float2(q.x, q.y), in, make_float2(q.z, q.w));
            }
            if (warp == ender) {
                end = in;
                for (int k = part; k >= 0; --k) {
                    const float4 q = meet.meeting.parts[slot][k][lane];
                    end = through<CUT>(make_float2(q.x, q.y), end, make_float2(q.z, q.w));
                }
                meet.carry[slot][lane] = end;
            }
            in = through<CUT>(P_in, in, own);
        };
        if (a.starts) meet_others(std::true_type{});
        else meet_others(std::false_type{});
        if (!met) {
            in = end = no_value();
            if (warp == ender) meet.carry[slot][lane] = end;
        }
        auto spread = [&](auto is_plain) {
            constexpr bool PLAIN = decltype(is_plain)::value;
#pragma unroll
            for (int j = 0; j < kTok; ++j) {
                if (!PLAIN && j >= have) continue;
                const bool start = !PLAIN && (starts >> j & 1);
                const float2 bj = mul2(to_x[j], input<0>(rows, j, lane));
                to_r[j] = start ? dup(0.0f) : UNIT ? fma2(to_r[j], pairs.minus_one, mul2(sg[j], state)) : mul2(sg[j], state);
                state = fma2(bj, pairs.minus_one, start ? dup(0.0f) : fade<PLAIN>(state, c[j], far >> 2 * j));
            }
            auto put = [&](int k, void* out, int j, float2 v) {
                if constexpr (TILE && PACK) put_row2<IO>(outs->g[k][j], lane, v);
                else if constexpr (TILE) put_row2<IO>(rows.in[k][j], lane, v);
                else store2<IO>(out, seq + (t0 + j) * (int64_t)D + c0, n, pair, v);
            };
#pragma unroll
            for (int j = kTok - 1; j >= 0; --j) {
                if (!PLAIN && j >= have) continue;
                const bool start = !PLAIN && (starts >> j & 1);
                in = add2(in, row2<IO>(rows.d_h[j], lane));
                const float2 minus = mul2(in, pairs.minus_one);
                put(0, ba.d_x, j, mul2(minus, to_x[j]));
                if (GATE) put(2, ba.d_g, j, mul2(minus, meet.stash[warp][j][lane]));
                in = start ? dup(0.0f) : fade<PLAIN>(in, c[j], far >> 2 * j);  // a lam
                const float2 dl = start ? dup(0.0f) : mul2(in, to_r[j]);      // d_log_a sg
                sum = add2(sum, dl);
                put(1, ba.d_r, j, start ? dl : mul2(dl, to_a[j]));  // a start's logit is not used, and may be a NaN
            }
        };
        if (plain) spread(std::true_type{});
        else spread(std::false_type{});
        if constexpr (TILE) {
            sm100::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0 && have > 0) {
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    const IO* from = nullptr;
                    if constexpr (PACK) from = outs->g[k][0];
                    else from = rows.in[k][0];
                    tile_store(&maps.out[k], first, t0, (int)b, from);
                }
                bulk_commit();
            }
        } else {
            __syncwarp();
            load((turn - 2) * parts + part, slot);
        }
    }
    if (part == 0 && warp == ender) store2<float>(ba.dh_init, b * D + c0, n, false, end);
    __syncthreads();
    meet.ends[0][warp][lane] = make_float2(-sum.x, -sum.y);
    __syncthreads();
    if (TILE) bulk_done();
    else copy_wait<0>();
    if (parts > 1 && !met) sm100::cluster_sync();  // the others may not be done sending; whoever is has left, or comes here too
    if (warp != 0) return;
    sum = meet.ends[0][0][lane];
    for (int w = 1; w < kWarps; ++w) sum = add2(sum, meet.ends[0][w][lane]);
    store2<float>(ba.part, (b * parts + part) * D + c0, n, false, sum);
}

// d_rate: the sums of all sequences and parts, in an order that depends on their number alone
__global__ void __launch_bounds__(256) scan_rate_kernel(const float* part, float* d_rate, const int64_t rows, const int D) {
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // it is launched beside the end of the reverse pass, and reads only when that is done
    float y = 0.0f;
    if (c < D)
        for (int64_t i = warp; i < rows; i += 8) y += part[i * D + c];
    sums[warp][lane] = y;
    __syncthreads();
    if (warp != 0 || c >= D) return;
    for (int w = 1; w < 8; ++w) y += sums[w][lane];
    d_rate[c] = y;
}

template <typename IO, bool GATE, bool UNIT, bool PACK, bool TILE> int launch(const ScanBwdArgs& b, const ScanMaps& maps, int by, bool pair, cudaStream_t st) {
    auto kernel = scan_bwd_kernel<IO, GATE, UNIT, PACK, TILE>;
    cudaError_t e = allow_shared_memory<scan_bwd_kernel<IO, GATE, UNIT, PACK, TILE>>();
    if (e != cudaSuccess) return (int)e;
    const ScanShape& s = b.f.s;
    const int parts = scan_bwd_parts(s);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.B * s.blocks() * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kMeet + kStages * kWarps * sizeof(Rows<IO, GATE ? 3 : 2, PACK>) + (PACK ? kWarps * sizeof(Outs<IO, GATE ? 3 : 2, true>) : 0);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kernel, b, maps, by, pair, parts);
    if (e != cudaSuccess) return (int)e;
    cudaLaunchConfig_t sum{};
    sum.gridDim = dim3((unsigned)((s.D + 31) / 32));
    sum.blockDim = dim3(256);
    sum.stream = st;
    at[0] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    sum.attrs = at;
    sum.numAttrs = 1;
    return (int)cudaLaunchKernelEx(&sum, scan_rate_kernel, (const float*)b.part, b.d_rate, (int64_t)s.B * parts, s.D);
}
template <typename IO, bool GATE, bool UNIT, bool PACK> int launch(const ScanBwdArgs& b, int by, bool pair, cudaStream_t st) {
    ScanMaps maps{};
    const void* in[4] = {b.f.x, b.f.r, b.f.g, b.d_h};
    for (int k = PACK ? 3 : 0; by == kByTile && k < 4; ++k)
        if (in[k] && !scan_map(&maps.in[k], in[k], b.f.s, kTok)) by = kBy4;
    const void* out[3] = {b.d_x, b.d_r, b.d_g};
    for (int k = 0; by == kByTile && k < (GATE ? 3 : 2); ++k)
        if (!scan_map(&maps.out[k], out[k], b.f.s, kTok)) by = kBy4;
    return by == kByTile ? launch<IO, GATE, UNIT, PACK, true>(b, maps, by, pair, st) : launch<IO, GATE, UNIT, PACK, false>(b, maps, by, pair, st);
}
template <typename IO, bool GATE, bool UNIT> int launch(const ScanBwdArgs& b, int by, bool pair, cudaStream_t st) {
    return b.f.codes ? launch<IO, GATE, UNIT, true>(b, by, pair, st) : launch<IO, GATE, UNIT, false>(b, by, pair, st);
}
template <typename IO> int dispatch(const ScanBwdArgs& b, int by, bool pair, cudaStream_t st) {
    if (b.f.s.gate) return b.f.s.unit ? launch<IO, true, true>(b, by, pair, st) : launch<IO, true, false>(b, by, pair, st);
    return b.f.s.unit ? launch<IO, false, true>(b, by, pair, st) : launch<IO, false, false>(b, by, pair, st);
}

}  // namespace

int scan_bwd_parts(const ScanShape& s) { return scan_parts(s, kTile, s.f32 ? 1 : 2); }

int scan_bwd_launch(const ScanBwdArgs& b, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    uintptr_t in = reinterpret_cast<uintptr_t>(b.d_h), out = 0;
    if (!b.f.codes) in |= reinterpret_cast<uintptr_t>(b.f.x) | reinterpret_cast<uintptr_t>(b.f.r) | reinterpret_cast<uintptr_t>(b.f.g);
    for (const void* p : {b.d_x, b.d_r, b.d_g}) out |= reinterpret_cast<uintptr_t>(p);
    int by = reads_by(b.f.s.D, b.f.s.f32, in);
    if (by == kByTile && out % 16 != 0) by = kBy4;
    const bool pair = b.f.s.D % 2 == 0 && out % (b.f.s.f32 ? 8 : 4) == 0;
    return b.f.s.f32 ? dispatch<float>(b, by, pair, st) : dispatch<__nv_bfloat16>(b, by, pair, st);
}

}  // namespace e2ttt
