// Gated linear recurrence, forward.  h_t = a_t h_{t-1} + b_t is linear in the state: over a run of tokens h_out = P h_in + h', P the product of the a_t and h' the run's
// end from a zero state.  A CTA has 64 channels of a sequence; a lane has two of them, a warp 16 tokens (fp32: 8) of a tile, whose P and h' meet in shared memory.  Where there are
// few channels and sequences, the tiles of a sequence are dealt out to the CTAs of a cluster, whose P and h' meet through distributed shared memory: no CTA waits for another
// cluster's work, nothing lies in global memory between them, and every sum has one order.
// A token's P and h' stay in registers from the walk to the output, so that gates are computed once; x, the logits and h go through shared memory by the copy engine, a warp's own
// rows at a time (loads by the threads themselves waited for places in the load queue: 87 us where the copy engine, all else being equal, took 74).
// 16384 tokens of 2048 in bf16 with an input gate: 64 us (268 MB, 4.2 TB/s, 64 % of the copy), 91 with rates of up to 4, whose decays take the exponential beside the series; with
// inputs kept in 8 bits 86 us; one sequence of 32768: 127 us; fp32 137 us (537 MB, 3.9 TB/s).  Rows that the copy engine cannot read: 160 us for 2046 channels, 295 for 2047.
// What bounds it: registers and shared memory allow two CTAs on an SM, and what these issue between their meetings (60 instructions and 8 special functions for a pair of values:
// 43 % of the issue slots, 53 % of the special function unit).
#include <type_traits>

#include "api_checks.h"
#include "pack8.cuh"
#include "scan_common.cuh"
#include "scan_map.h"

namespace e2ttt {
namespace {
using namespace scan;

constexpr int kStages = 2;
template <typename IO> constexpr int kTokOf = sizeof(IO) == 2 ? 16 : 8;

// what the warps of a tile and the parts of a cluster leave for one another, twice in turn
struct Meet {
    float4 runs[2][kWarps][32];  // P and h' of a warp's tokens
    float2 carry[2][32];         // the state after a turn's tokens
    uint64_t full[kWarps][kStages];
    Meeting meeting;
};

constexpr int kMeet = (sizeof(Meet) + 127) / 128 * 128;

// The 8-bit form of a warp's rows of one tensor: a lane takes 32 bytes, half a block in bf16 and a quarter of one in fp32, and writes their codes at once.
template <typename IO, int ROWS, bool LOGIT> __device__ __forceinline__ void pack_rows(const IO* rows, uint8_t* codes, uint8_t* scales, int n, int lane) {
    constexpr int V = 32 / (int)sizeof(IO), PER = kScanCh / V, STEP = 32 / PER;  // lanes of a row; rows a warp takes at once
    const int row = lane / PER, chunk = lane % PER;
#pragma unroll
    for (int i = 0; i < ROWS; i += STEP) {
        struct alignas(16) Piece {
            IO x[V];
        };
        const Piece p = *reinterpret_cast<const Piece*>(rows + (row + i) * kScanCh + chunk * V);
        uint32_t byte;
        const pack8::Codes<V> code = pack8::encode<IO, V, LOGIT>(p.x, pack8::group_magnitude<IO, V>(p.x), byte);
        if (row + i >= n) continue;
        *reinterpret_cast<pack8::Codes<V>*>(codes + (row + i) * kScanCh + chunk * V) = code;
        if (chunk % (pack8::kBlock / V) == 0) scales[(row + i) * 2 + chunk / (pack8::kBlock / V)] = (uint8_t)byte;
    }
}

// TILE: rows are read by kByTile
template <typename IO, bool GATE, bool UNIT, bool PACK, bool TILE>
__global__ void __launch_bounds__(kThreads, 2) scan_fwd_kernel(const ScanArgs a, const __grid_constant__ ScanMaps maps, const int by, const bool pair, const int parts) {
    constexpr int TOK = kTokOf<IO>, kTile = TOK * kWarps, NT = GATE ? 3 : 2;
    extern __shared__ __align__(128) char smem[];
    Meet& meet = *reinterpret_cast<Meet*>(smem);
    const int D = a.s.D, L = a.s.L, lane = threadIdx.x & 31, warp = __shfl_sync(kAll, threadIdx.x >> 5, 0);
    const int64_t blocks = a.s.blocks(), spans = a.s.spans(), unit = blockIdx.x / parts, b = unit / blocks;
    const int part = blockIdx.x - (int)(unit * parts), first = (int)(unit - b * blocks) * kScanCh;
    const int c0 = first + 2 * lane, n = max(0, min(2, D - c0));
    const bool whole = first + kScanCh <= D;  // all channels are there
    IO* ring = reinterpret_cast<IO*>(smem + kMeet) + warp * (kStages * NT * TOK * kScanCh);
    const int64_t seq = b * L * (int64_t)D;
    const Pairs pairs = make_pairs();
    float2 rate = load2<float>(a.rate, c0, n, false);
    const bool near = __syncthreads_and(whole && near_rate(rate.x) && near_rate(rate.y));
    rate = make_float2(-rate.x, -rate.y);
    float2 end = a.h_init ? load2<float>(a.h_init, b * D + c0, n, false) : dup(0.0f);  // the state after the last turn, in one warp
    const int ender = parts == 1 ? kWarps - 1 : 0;
    if (warp == ender) meet.carry[1][lane] = end;
    uint64_t* full = meet.full[warp];
    if (TILE && lane == 0) {
        for (int i = 0; i < kStages; ++i) sm100::mbar_init(&full[i], 1);
        sm100::fence_mbar_init();
    }
    __syncwarp();
    if (parts > 1) meeting_init(meet.meeting);
    const int64_t tiles = ((int64_t)L + kTile - 1) / kTile;
    auto has_rows = [&](int64_t tile) { return tile * kTile + warp * TOK < L; };
    unsigned next_first = 0;
    bool met = true;  // no wait of this warp has given up
    auto load = [&](int64_t tile, int slot) {
        next_first = 0;
        if ((!TILE || met) && has_rows(tile)) {
            const int t = (int)(tile * kTile) + warp * TOK;
            IO* to = ring + slot * (NT * TOK * kScanCh);
            if constexpr (TILE) {
                if (lane == 0) {
                    sm100::mbar_expect_tx(&full[slot], NT * TOK * kScanCh * sizeof(IO));
#pragma unroll
                    for (int k = 0; k < NT; ++k) tile_load(to + k * TOK * kScanCh, &maps.in[k], first, t, (int)b, &full[slot]);
                }
            } else {
                copy_rows<IO, TOK>(to, static_cast<const IO*>(a.x), seq, t, L, first, D, by, lane);
                copy_rows<IO, TOK>(to + TOK * kScanCh, static_cast<const IO*>(a.r), seq, t, L, first, D, by, lane);
                if (GATE) copy_rows<IO, TOK>(to + 2 * TOK * kScanCh, static_cast<const IO*>(a.g), seq, t, L, first, D, by, lane);
            }
            if (a.starts && lane < TOK && t + lane < L) next_first = a.starts[b * L + t + lane];
        }
        if (!TILE) copy_commit();
    };
    load(part, 0);
    unsigned byte0 = next_first;
    load(part + parts, 1);
    int slot = 0;
    uint32_t parity = 0;
    auto give_up = [&](bool next) {  // next: the next turn's rows are under way
        met = false;
        if constexpr (TILE) {
            if (next) (void)await_on<false>(&full[slot ^ 1], parity ^ (uint32_t)slot, sm100::kWaitCycles);
            if (lane == 0) bulk_read_done();
            __syncwarp();
            fill(ring, kNans, kStages * NT * TOK * kScanCh * (int)sizeof(IO));
        }
    };
    // every CTA of a cluster takes every turn: its part of the last one may be empty
    for (int64_t turn = 0; turn * parts < tiles; ++turn, slot ^= 1, parity ^= slot == 0) {
        const int64_t tile = turn * parts + part;
        const int t0 = (int)min(tile * kTile + warp * TOK, (int64_t)L), have = min(TOK, L - t0);
        const unsigned starts = __ballot_sync(kAll, byte0 != 0);
        byte0 = next_first;
        IO* rows = ring + slot * (NT * TOK * kScanCh);
        if (!TILE) {
            copy_wait<kStages - 1>();
        } else if (met && have > 0 && !await<false>(&full[slot], parity, a.wait_cycles)) {
            (void)await_on<false>(&full[slot], parity, sm100::kWaitCycles);
            give_up(turn == 0 && has_rows(tile + parts));
        }
        __syncwarp();
        if (PACK && have > 0) {
            const int64_t row = unit * spans * kScanSpan + t0;
            uint8_t *codes = a.codes + row * kScanCh, *scales = a.scales + row * 2;
            pack_rows<IO, TOK, false>(rows, codes, scales, have, lane);
#pragma unroll
            for (int k = 1; k < NT; ++k) pack_rows<IO, TOK, true>(rows + k * TOK * kScanCh, codes + k * a.code_step, scales + k * a.scale_step, have, lane);
        }
        float2 h[TOK], P[TOK], hh = dup(0.0f), pp = dup(1.0f);
        const bool plain = near && have == TOK && !starts;  // all tokens and channels are there, none is a start, no decay is far from 1
        auto walk = [&](auto is_plain) {
            constexpr bool PLAIN = decltype(is_plain)::value;
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                if (PLAIN || j < have) {
                    float2 u = row2(rows + j * kScanCh, lane), sg;
                    if constexpr (GATE) {
                        float2 ig, r = logit2(rows + (TOK + j) * kScanCh, lane);
                        if (!PLAIN && (starts >> j & 1)) r = no_nan(r);
                        sigmoids<IO>(pairs, r, logit2(rows + (2 * TOK + j) * kScanCh, lane), sg, ig);
                        u = mul2(u, ig);
                    } else {
                        sg = sigmoid2<IO>(pairs, logit2(rows + (TOK + j) * kScanCh, lane));
                    }
                    const Decay d = decay<IO, UNIT, PLAIN>(pairs, sg, rate);
                    if (!PLAIN && (starts >> j & 1)) {
                        hh = u;
                    } else {
                        if (UNIT) u = mul2(u, sqrt_minus(d.minus));
                        hh = add2(fade<PLAIN>(hh, d.c, d.far), u);
                        pp = fade<PLAIN>(pp, d.c, d.far);
                    }
                }
                h[j] = hh;
                P[j] = !PLAIN && cut_by(starts, j) ? dup(kCut) : pp;
            }
            pp = P[TOK - 1];
        };
        if (plain) walk(std::true_type{});
        else walk(std::false_type{});
        __syncwarp();
        if constexpr (!TILE) {
            load((turn + 2) * parts + part, slot);
        } else if (turn != 0) {  // the last turn's states have left its stage by now
            if (lane == 0) bulk_read_done();
            __syncwarp();
            load((turn + 1) * parts + part, slot ^ 1);
            byte0 = next_first;
        }
        meet.runs[slot][warp][lane] = make_float4(pp.x, pp.y, hh.x, hh.y);
        __syncthreads();
        const float2 before = meet.carry[slot ^ 1][lane];  // the state before the turn's tokens
        float2 in = before;
        auto meet_others = [&](auto is_cut) {
            constexpr bool CUT = decltype(is_cut)::value;
            if (parts == 1) {
#pragma unroll
                for (int w = 0; w < kWarps - 1; ++w) {
                    if (w >= warp) break;
                    const float4 q = meet.runs[slot][w][lane];
                    in = through<CUT>(make_float2(q.x, q.y), in, make_float2(q.z, q.w));
                }
                if (warp == ender) meet.carry[slot][lane] = end = through<CUT>(pp, in, hh);
                return;
            }
            float2 P_in = dup(1.0f), own = dup(0.0f);  // the warps before this one
#pragma unroll
            for (int w = 0; w < kWarps - 1; ++w) {
                if (w >= warp) break;
                const float4 q = meet.runs[slot][w][lane];
                own = through<CUT>(make_float2(q.x, q.y), own, make_float2(q.z, q.w));
                P_in = both<CUT>(P_in, make_float2(q.x, q.y));
            }
            if (warp == kWarps - 1 && met) send_part(meet.meeting, slot, part, parts, lane, both<CUT>(P_in, pp), through<CUT>(pp, own, hh));
            if (met && !await<true>(&meet.meeting.full[slot], parity, a.wait_cycles)) {
                (void)await_on<true>(&meet.meeting.full[slot], parity, kSendCycles);
                give_up(has_rows(tile + parts));
            }
            for (int k = 0; k < part; ++k) {
                const float4 q = meet.meeting.parts[slot][k][lane];
                in = through<CUT>(make_float2(q.x, q.y), in, make_float2(q.z, q.w));
            }
            if (warp == ender) {
                end = in;
                for (int k = part; k < parts; ++k) {
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
        if (a.states && have > 0 && t0 % kScanSpan == 0) store2<float>(a.states, (b * spans + t0 / kScanSpan) * D + c0, n, false, in);
        if (!a.h) continue;
        if constexpr (TILE) {  // in the place of x
            if (plain) {
#pragma unroll
                for (int j = 0; j < TOK; ++j) put_row2<IO>(rows + j * kScanCh, lane, fma2(P[j], in, h[j]));
            } else {
#pragma unroll
                for (int j = 0; j < TOK; ++j)
                    if (j < have) put_row2<IO>(rows + j * kScanCh, lane, through<true>(P[j], in, h[j]));
            }
            sm100::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0 && have > 0) {
                tile_store(&maps.out[0], first, t0, (int)b, rows);
                bulk_commit();
            }
        } else {
            const int64_t at = seq + (int64_t)t0 * D + c0;
#pragma unroll
            for (int j = 0; j < TOK; ++j)
                if (j < have) store2<IO>(a.h, at + j * (int64_t)D, n, pair, through<true>(P[j], in, h[j]));
        }
    }
    if (a.h_final && part == 0 && warp == ender) store2<float>(a.h_final, b * D + c0, n, false, end);
    if (TILE) bulk_done();
    else copy_wait<0>();
    if (parts > 1 && !met) sm100::cluster_sync();  // the others may not be done sending; whoever is has left, or comes here too
}

// CTAs of a cluster
int parts_of(const ScanShape& s) { return scan_parts(s, (s.f32 ? kTokOf<float> : kTokOf<__nv_bfloat16>) * kWarps, 2); }

template <typename IO, bool GATE, bool UNIT, bool PACK, bool TILE> int launch(const ScanArgs& a, const ScanMaps& maps, int by, bool pair, cudaStream_t st) {
    auto kernel = scan_fwd_kernel<IO, GATE, UNIT, PACK, TILE>;
    cudaError_t e = allow_shared_memory<scan_fwd_kernel<IO, GATE, UNIT, PACK, TILE>>();
    if (e != cudaSuccess) return (int)e;
    const int parts = parts_of(a.s);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.s.B * a.s.blocks() * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kMeet + kStages * (GATE ? 3 : 2) * kTokOf<IO> * kWarps * kScanCh * sizeof(IO);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    return (int)cudaLaunchKernelEx(&cfg, kernel, a, maps, by, pair, parts);
}
template <typename IO, bool GATE, bool UNIT, bool PACK> int launch(const ScanArgs& a, int by, bool pair, cudaStream_t st) {
    ScanMaps maps{};
    const void* in[3] = {a.x, a.r, a.g};
    for (int k = 0; by == kByTile && k < (GATE ? 3 : 2); ++k)
        if (!scan_map(&maps.in[k], in[k], a.s, kTokOf<IO>)) by = kBy4;
    if (by == kByTile && a.h && !scan_map(&maps.out[0], a.h, a.s, kTokOf<IO>)) by = kBy4;
    return by == kByTile ? launch<IO, GATE, UNIT, PACK, true>(a, maps, by, pair, st) : launch<IO, GATE, UNIT, PACK, false>(a, maps, by, pair, st);
}
template <typename IO, bool GATE, bool UNIT> int launch(const ScanArgs& a, int by, bool pair, cudaStream_t st) {
    return a.codes ? launch<IO, GATE, UNIT, true>(a, by, pair, st) : launch<IO, GATE, UNIT, false>(a, by, pair, st);
}
template <typename IO> int dispatch(const ScanArgs& a, int by, bool pair, cudaStream_t st) {
    if (a.s.gate) return a.s.unit ? launch<IO, true, true>(a, by, pair, st) : launch<IO, true, false>(a, by, pair, st);
    return a.s.unit ? launch<IO, false, true>(a, by, pair, st) : launch<IO, false, false>(a, by, pair, st);
}

}  // namespace

int scan_fwd_launch(const ScanArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const uintptr_t in = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.r) | reinterpret_cast<uintptr_t>(a.g);
    int by = reads_by(a.s.D, a.s.f32, in);
    if (by == kByTile && reinterpret_cast<uintptr_t>(a.h) % 16 != 0) by = kBy4;
    const bool pair = a.s.D % 2 == 0 && reinterpret_cast<uintptr_t>(a.h) % (a.s.f32 ? 8 : 4) == 0;
    return a.s.f32 ? dispatch<float>(a, by, pair, st) : dispatch<__nv_bfloat16>(a, by, pair, st);
}

}  // namespace e2ttt
