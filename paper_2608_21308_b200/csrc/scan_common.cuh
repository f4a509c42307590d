// Gated linear recurrence: the gates of a token, two channels at a time, and the tokens of a thread.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "scan.h"
#include "sm100.cuh"

namespace e2ttt {
namespace scan {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;

// two fp32 values at a time (one instruction on this architecture)
__device__ __forceinline__ uint64_t u2(float2 a) { return *reinterpret_cast<const uint64_t*>(&a); }
__device__ __forceinline__ float2 f2(uint64_t a) { return *reinterpret_cast<const float2*>(&a); }
__device__ __forceinline__ float2 dup(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 no_value() { return dup(__uint_as_float(0x7fc00000u)); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(u2(a)), "l"(u2(b)), "l"(u2(c)));
    return f2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(u2(a)), "l"(u2(b)));
    return f2(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(u2(a)), "l"(u2(b)));
    return f2(r);
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rsqrt_fast(float x) {
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float kLog2e = 1.4426950408889634f;

// Constants of the gates as pairs, moved to registers by hand so that they are there once
struct Pairs {
    float2 neg_log2e, one, two, minus_one, e1, e2, e3, e4;
};
__device__ __forceinline__ float2 kept(float x) {
    float y;
    asm volatile("mov.b32 %0, %1;" : "=f"(y) : "f"(x));
    return dup(y);
}
// (exp(y) - 1) / y = 1 + e1 y + .. + e4 y^4 on [-1/4, 0], fitted to the least largest relative error: 2.9e-9
__device__ __forceinline__ Pairs make_pairs() {
    return Pairs{kept(-kLog2e), kept(1.0f), kept(2.0f), kept(-1.0f), kept(0.49999964f), kept(0.16665289f), kept(0.04150013f), kept(0.00753017f)};
}

// Logits count from -43 on: the product of two exp(-x) stays finite, and 1 - a^2 above 0 at any ordinary rate.  A NaN stays one.
constexpr float kLeast = -43.0f;  // also what 8-bit inputs hold
__device__ __forceinline__ float2 capped(float2 x) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(kLeast));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(kLeast));
    return x;
}
// exp(-x) of capped logits, for the sigmoid 1 / (1 + exp(-x)) and what it leaves of 1, exp(-x) / (1 + exp(-x)): an open gate's rest is computed, not subtracted.  With bf16 I/O
// the special function unit's 2^-22 is enough.
template <typename IO> __device__ __forceinline__ float2 exp_neg(const Pairs& k, float2 x) {
    if constexpr (sizeof(IO) == 4) return make_float2(expf(-x.x), expf(-x.y));
    const float2 t = mul2(x, k.neg_log2e);
    return make_float2(ex2(t.x), ex2(t.y));
}
template <typename IO> __device__ __forceinline__ float2 reciprocal(float2 x) {
    if constexpr (sizeof(IO) == 4) return make_float2(__frcp_rn(x.x), __frcp_rn(x.y));
    return make_float2(rcp(x.x), rcp(x.y));
}
template <typename IO> __device__ __forceinline__ float2 sigmoid2(const Pairs& k, float2 x) { return reciprocal<IO>(add2(exp_neg<IO>(k, x), k.one)); }
// the sigmoids of two pairs; with bf16 I/O one reciprocal of both denominators: the special function unit bounds the forward otherwise
template <typename IO> __device__ __forceinline__ void sigmoids(const Pairs& k, float2 x, float2 y, float2& sx, float2& sy) {
    if constexpr (sizeof(IO) == 4) {
        sx = sigmoid2<IO>(k, x);
        sy = sigmoid2<IO>(k, y);
    } else {
        const float2 p = add2(exp_neg<IO>(k, x), k.one), q = add2(exp_neg<IO>(k, y), k.one), r = reciprocal<IO>(mul2(p, q));
        sx = mul2(q, r);
        sy = mul2(p, r);
    }
}

// A token's decay for two channels.  Near 1, where a's own rounding is what a long memory adds up, it is kept as c = a - 1; far from it (log a below -1/4), where c's rounding
// would be what a leaves of a state, as c = a.  minus = a^2 - 1.
struct Decay {
    float2 c, minus;
    unsigned far;  // bit 0: the first channel's c is a, bit 1: the second's
};
// Whether a rate's decays are all near 1, and none of them 1
__device__ __forceinline__ bool near_rate(float rate) { return rate >= 1e-10f && rate <= 0.25f; }
// sg = sigmoid(a_decay).  NEAR: near_rate of both channels.
template <typename IO, bool UNIT, bool NEAR> __device__ __forceinline__ Decay decay(const Pairs& k, float2 sg, float2 neg_rate) {
    const float2 y = mul2(neg_rate, sg);
    Decay d;
    float2 p = fma2(y, k.e4, k.e3);
    p = fma2(p, y, k.e2);
    p = fma2(p, y, k.e1);
    p = fma2(p, y, k.one);
    d.c = mul2(p, y);
    d.far = 0;
    if (UNIT) d.minus = mul2(d.c, add2(d.c, k.two));
    if constexpr (!NEAR) {
        float2 e;
        if constexpr (sizeof(IO) == 4) e = make_float2(expf(y.x), expf(y.y));
        else e = make_float2(ex2(y.x * kLog2e), ex2(y.y * kLog2e));
        if (y.x < -0.25f) {
            d.far = 1;
            d.c.x = e.x;
            if (UNIT) d.minus.x = fmaf(e.x, e.x, -1.0f);
        }
        if (y.y < -0.25f) {
            d.far |= 2;
            d.c.y = e.y;
            if (UNIT) d.minus.y = fmaf(e.y, e.y, -1.0f);
        }
    }
    return d;
}
// a h
template <bool NEAR> __device__ __forceinline__ float2 fade(float2 h, float2 c, unsigned far) {
    if constexpr (NEAR) return fma2(h, c, h);
    return fma2(h, c, make_float2(far & 1 ? 0.0f : h.x, far & 2 ? 0.0f : h.y));
}
// sqrt(-x), and 1 / sqrt(-x) with 0 for 0; both good to 2^-22.  NEAR: x is not 0.
__device__ __forceinline__ float2 sqrt_minus(float2 x) {
    float2 y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(-x.x));
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(-x.y));
    return y;
}
template <bool NEAR> __device__ __forceinline__ float2 inv_sqrt_minus(float2 x) {
    const float2 y = make_float2(rsqrt_fast(-x.x), rsqrt_fast(-x.y));
    if constexpr (NEAR) return y;
    return make_float2(x.x < -1e-37f ? y.x : 0.0f, x.y < -1e-37f ? y.y : 0.0f);
}

template <typename IO> __device__ __forceinline__ float to_f32(IO x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Two neighbouring channels of a row; `n` of them are there.  `pair`: the row's channels lie at a multiple of the pair's size.
template <typename IO> __device__ __forceinline__ float2 load2(const void* base, int64_t at, int n, bool pair) {
    const IO* p = static_cast<const IO*>(base) + at;
    if (pair && n == 2) {
        if constexpr (sizeof(IO) == 4) {
            return *reinterpret_cast<const float2*>(p);
        } else {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
            return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        }
    }
    return make_float2(n > 0 ? to_f32<IO>(p[0]) : 0.0f, n > 1 ? to_f32<IO>(p[1]) : 0.0f);
}
template <typename IO> __device__ __forceinline__ void store2(void* base, int64_t at, int n, bool pair, float2 v) {
    IO* p = static_cast<IO*>(base) + at;
    if (pair && n == 2) {
        if constexpr (sizeof(IO) == 4) {
            *reinterpret_cast<float2*>(p) = v;
        } else {
            const __nv_bfloat162 w = __floats2bfloat162_rn(v.x, v.y);
            *reinterpret_cast<__nv_bfloat162*>(p) = w;
        }
        return;
    }
    if (n > 0) put(p, v.x);
    if (n > 1) put(p + 1, v.y);
}

// ---- a warp's tokens of a tile, ahead in shared memory: rows of 64 channels, one tensor after the other.  Every warp reads back only what it copied itself.
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(dst)), "l"(src) : "memory");
}
// 4 bytes, zeros where `in` is false (nothing is read then)
__device__ __forceinline__ void copy4(void* dst, const void* src, bool in) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_at(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
// tiles and contiguous pieces by the copy engine, counted on a barrier; what lies outside the tensor is filled with zeros
__device__ __forceinline__ void tile_load(void* dst, const void* map, int c, int t, int b, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_at(dst)), "l"(map), "r"(c), "r"(t),
                 "r"(b), "r"(smem_at(bar))
                 : "memory");
}
// a tile from shared memory; what lies outside the tensor is not written
__device__ __forceinline__ void tile_store(const void* map, int c, int t, int b, const void* src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(c), "r"(t), "r"(b), "r"(smem_at(src)) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_read_done() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }  // shared memory may be written again
__device__ __forceinline__ void bulk_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_at(dst)), "l"(src), "r"(bytes), "r"(smem_at(bar)) : "memory");
}

// How rows are read (fp32 always by one of the first two): tiles by the copy engine (addresses and row lengths that are a multiple of 16 bytes; one lane starts them, and no other instruction waits for a place in the
// load queue), pieces of 4 bytes, or value by value (odd rows, and addresses, of bf16)
enum { kByTile = 0, kBy4 = 1, kByValue = 2 };
inline int reads_by(int D, bool f32, uintptr_t all) {
    const int size = f32 ? 4 : 2;
    if (all % 16 == 0 && (int64_t)D * size % 16 == 0) return kByTile;
    return all % 4 == 0 && (int64_t)D * size % 4 == 0 ? kBy4 : kByValue;
}

// ROWS tokens of `src` from row t on, channels c .. c + 63, as far as there are tokens (L) and channels (D); `at` is where token 0 of the sequence starts
template <typename IO, int ROWS> __device__ __forceinline__ void copy_rows(IO* dst, const IO* src, int64_t at, int t, int L, int c, int D, int by, int lane) {
    const IO* from = src + (at + (int64_t)t * D + c);
    if (by == kBy4) {
        constexpr int V = 4 / (int)sizeof(IO), WORDS = kScanCh / V / 32;  // words of a row that a lane copies
#pragma unroll
        for (int h = 0; h < WORDS; ++h) {
            const int ch = (lane + 32 * h) * V;
            const IO* p = from + ch;
#pragma unroll
            for (int row = 0; row < ROWS; ++row, p += D) {
                const bool in = c + ch < D && t + row < L;
                copy4(dst + row * kScanCh + ch, in ? p : src, in);
            }
        }
        return;
    }
    if constexpr (sizeof(IO) == 2) {
        const IO* p = from + 2 * lane;
        const int n = D - c - 2 * lane;
        uint32_t w[ROWS];
#pragma unroll
        for (int row = 0; row < ROWS; ++row, p += D) {
            uint32_t x = 0, y = 0;
            if (t + row < L && n > 0) x = *reinterpret_cast<const uint16_t*>(p);
            if (t + row < L && n > 1) y = *reinterpret_cast<const uint16_t*>(p + 1);
            w[row] = x | y << 16;
        }
#pragma unroll
        for (int row = 0; row < ROWS; ++row) reinterpret_cast<uint32_t*>(dst + row * kScanCh)[lane] = w[row];
    }
}

// a lane's two channels of a row in shared memory
template <typename IO> __device__ __forceinline__ void put_row2(IO* row, int lane, float2 v) {
    if constexpr (sizeof(IO) == 4) reinterpret_cast<float2*>(row)[lane] = v;
    else reinterpret_cast<__nv_bfloat162*>(row)[lane] = __floats2bfloat162_rn(v.x, v.y);
}
template <typename IO> __device__ __forceinline__ float2 row2(const IO* row, int lane) {
    if constexpr (sizeof(IO) == 4) {
        return reinterpret_cast<const float2*>(row)[lane];
    } else {
        const uint32_t w = reinterpret_cast<const uint32_t*>(row)[lane];
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
}

// the same of a logit, capped
template <typename IO> __device__ __forceinline__ float2 logit2(const IO* row, int lane) {
    if constexpr (sizeof(IO) == 4) {
        return capped(row2(row, lane));
    } else {
        const __nv_bfloat162 w = __hmax2_nan(reinterpret_cast<const __nv_bfloat162*>(row)[lane], __float2bfloat162_rn(kLeast));
        const uint32_t u = *reinterpret_cast<const uint32_t*>(&w);
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
}

// A start's decay logit: it is not used, but its sigmoid may share a reciprocal with the input gate's, which a NaN would reach
__device__ __forceinline__ float2 no_nan(float2 logit) { return make_float2(fmaxf(logit.x, kLeast), fmaxf(logit.y, kLeast)); }

// ---- runs of tokens: what goes in, P times, plus what a run makes of nothing.  CUT: there are starts, and a run with one in it lets nothing through, an infinity or a NaN
// neither.  Such a run has kCut for its P: a product of decays is never negative, but 0 where it underflows, and a NaN behind the start where a logit is one.
constexpr float kCut = -1.0f;
template <bool CUT> __device__ __forceinline__ float2 through(float2 P, float2 in, float2 own) {
    if constexpr (!CUT) return fma2(P, in, own);
    return make_float2(P.x < 0.0f ? own.x : fmaf(P.x, in.x, own.x), P.y < 0.0f ? own.y : fmaf(P.y, in.y, own.y));
}
// P of two runs
template <bool CUT> __device__ __forceinline__ float2 both(float2 P, float2 next) {
    if constexpr (!CUT) return mul2(P, next);
    return make_float2(P.x < 0.0f || next.x < 0.0f ? kCut : P.x * next.x, P.y < 0.0f || next.y < 0.0f ? kCut : P.y * next.y);
}
// whether one of a run's tokens up to the j-th is a start
__device__ __forceinline__ bool cut_by(unsigned starts, int j) { return (starts & ((2u << j) - 1)) != 0; }

// ---- CTAs of a cluster: the parts of a sequence's channels along its tokens.  Every turn each leaves its tile's run with all of them by asynchronous stores, which count
// themselves on the receiver's barrier (a release of the CTA's global stores, as a cluster's barrier takes, would wait for all of them).  A buffer is used again two turns later: a CTA
// sends there only after all others have sent what follows it, which they do when their warps have read it.
struct Meeting {
    float4 parts[2][8][32];  // P and what a tile makes of nothing, of every CTA
    uint64_t full[2];
};
__device__ __forceinline__ void meeting_init(Meeting& m) {
    if (threadIdx.x == 0) {
        sm100::mbar_init(&m.full[0], 1);
        sm100::mbar_init(&m.full[1], 1);
        sm100::fence_mbar_init();
    }
    sm100::cluster_sync();  // the others' shared memory is there
}
__device__ __forceinline__ uint32_t in_cta(uint32_t at, uint32_t rank) {
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    return there;
}
// one warp sends
__device__ __forceinline__ void send_part(Meeting& m, int slot, int part, int parts, int lane, float2 P, float2 own) {
    if (lane == 0) sm100::mbar_expect_tx(&m.full[slot], parts * 512);
    __syncwarp();
    const uint32_t data = smem_at(&m.parts[slot][part][lane]), bar = smem_at(&m.full[slot]);
    for (int k = 0; k < parts; ++k)
        sm100::st_async_v4(in_cta(data, k), __float_as_uint(P.x), __float_as_uint(P.y), __float_as_uint(own.x), __float_as_uint(own.y), in_cta(bar, k));
}
// ---- waits that give up.  Every wait is bounded, by `limit` cycles (0: it gives up without a look), though neither the copies nor the stores of a cluster can fail short of a
// device fault.  A warp that gives up waits once more for what is under way to its shared memory, has NaNs for rows from then on, and neither loads, waits nor sends any more: what it
// computes and hands on is NaN, and the waits of CTAs that it does not send to give up too.
template <bool CLUSTER> __device__ __noinline__ bool await_on(uint64_t* bar, uint32_t parity, long long limit) {
    const long long t0 = clock64();
    while (!__any_sync(kAll, clock64() - t0 >= limit))
        if (__all_sync(kAll, sm100::mbar_try_wait<CLUSTER>(bar, parity))) return true;
    return false;
}
// the whole warp calls, and gets one answer
template <bool CLUSTER> __device__ __forceinline__ bool await(uint64_t* bar, uint32_t parity, long long limit) {
    return __all_sync(kAll, limit != 0 && sm100::mbar_try_wait<CLUSTER>(bar, parity)) || await_on<CLUSTER>(bar, parity, limit);
}
constexpr long long kSendCycles = 100000;  // a store to another CTA takes some thousand
// a warp's bytes in shared memory, 16 at a time
static __device__ __noinline__ void fill(void* at, uint32_t word, int bytes) {
    const int lane = threadIdx.x & 31;
    for (int i = lane; i < bytes / 16; i += 32) static_cast<uint4*>(at)[i] = make_uint4(word, word, word, word);
    __syncwarp();
}
constexpr uint32_t kNans = 0xffffffffu;  // in either type, and for the scales of packed rows

}  // namespace scan
}  // namespace e2ttt
