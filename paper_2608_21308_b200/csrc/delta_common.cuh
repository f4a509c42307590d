// Gated delta rule: fragments, the two-term fp16 form of an operand, tile addressing.
//
// Products run as mma.m16n8k16 with fp16 operands and fp32 sums.  A state is cut into slices of 16 value rows, one warp each: the slice
// stays in a warp's accumulators for the whole sequence, an accumulator tile is the next product's A operand as it is, and no value
// crosses a warp.  Measured on B200: an m16n8k16 takes 8.1 cycles of its scheduler (1024 multiply-adds per cycle and SM), its result 21, and
// other arithmetic does not run beside it (one MMA and four FMAs take 12.1 cycles, with six 14.1), so a chain of dependent chunks is bound by what
// its warp issues.  A 128-row tensor-memory tile would hold one sequence per SM (64 sequences: 64 of 148 SMs; a 64-row tile half of one), and send the state through tensor
// memory and back, and through the splitting into terms, between any two of the four dependent products of a chunk.
// Operands in 32 bits are used as two fp16 terms, x = 2^-s (hi + lo): 22 bits, and s (a power of two per slice or tile, from its largest
// value or a bound on it) keeps both terms inside fp16's exponents.  What is bf16 on input is one term, exactly down to 2^-24 of its tile's largest
// value.  (Two bf16 terms, 16 bits, leave 3e-6 in every product: the fp32 outputs would be ten times less exact.)
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "delta.h"
#include "sm100.cuh"

namespace e2ttt {
namespace delta {

constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename IO> __device__ __forceinline__ IO from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// power of two that brings a largest magnitude m into [2^12, 2^13) (2^100 at most: m = 0), and its inverse
__device__ __forceinline__ void pow2_scale(float m, float& s, float& inv) {
    int e = 139 - (int)(__float_as_uint(m) >> 23);
    e = max(-100, min(100, e));
    s = __uint_as_float((uint32_t)(127 + e) << 23);
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
}
// the same from a bound on the magnitudes: [2^13, 2^14), a factor of four below fp16's largest value.  A bound may be 2^10 above what it bounds:
// the second term's smallest step, 2^-24, is then still 2^-27 of the largest value.
__device__ __forceinline__ void pow2_bound(float m, float& s, float& inv) {
    int e = 140 - (int)(__float_as_uint(m) >> 23);
    e = max(-100, min(100, e));
    s = __uint_as_float((uint32_t)(127 + e) << 23);
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
}
// Product of two scales that meets a sum of zeros wherever it is this large (a bound of 0 has the scale 2^100: a state of 2^28 or more beside a chunk without keys
// and values): kept finite, so that zeros stay zeros.
__device__ __forceinline__ float scales(float x, float y) { return fminf(x * y, 0x1p120f); }
// two fp32 values at a time (one instruction on this architecture)
__device__ __forceinline__ uint64_t pack2(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t p, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b0, float b1, float c0, float c1) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pack2(a0, a1)), "l"(pack2(b0, b1)), "l"(pack2(c0, c1)));
    unpack2(r, d0, d1);
}
__device__ __forceinline__ void mul2(float& d0, float& d1, float a0, float a1, float b0, float b1) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a0, a1)), "l"(pack2(b0, b1)));
    unpack2(r, d0, d1);
}
__device__ __forceinline__ void add2(float& d0, float& d1, float a0, float a1) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(d0, d1)), "l"(pack2(a0, a1)));
    unpack2(r, d0, d1);
}
__device__ __forceinline__ float warp_sum(float m) {
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) m += __shfl_xor_sync(kAll, m, i);
    return m;
}
__device__ __forceinline__ float warp_max(float m) {
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, i));
    return m;
}

__device__ __forceinline__ uint32_t pack_half(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(x, y);
    const float2 f = __half22float2(h);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    float r, q;
    fma2(r, q, f.x, f.y, -1.0f, -1.0f, x, y);
    lo = pack_half(r, q);
}
// the two values of a word of first and of second terms
__device__ __forceinline__ void join_terms(uint32_t hi, uint32_t lo, float& x, float& y) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi)), e = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    x = f.x + e.x;
    y = f.y + e.y;
}
// Eight values of a term brought to another scale by a power of two, at most 1: below 2^-14 that power has fewer bits in fp16 than the values that it leaves, or none.
__device__ __forceinline__ uint4 times_ratio(const uint4& x, float ratio) {
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    if (ratio >= 0x1p-14f) {
        const __half2 m = __float2half2_rn(ratio);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&w[i]), m);
            w[i] = *reinterpret_cast<const uint32_t*>(&z);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            w[i] = pack_half(f.x * ratio, f.y * ratio);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// an operand that carries its scale already
__device__ __forceinline__ void split_a(const float (&x)[4], const float (&y)[4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    split(x[0], x[1], hi[0], lo[0]);
    split(x[2], x[3], hi[1], lo[1]);
    split(y[0], y[1], hi[2], lo[2]);
    split(y[2], y[3], hi[3], lo[3]);
}

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same without a sum to start from
__device__ __forceinline__ void mma0(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
// largest of the lanes' values, none negative: their bits are ordered as they are
__device__ __forceinline__ float warp_most(float x) {
    return __uint_as_float(__reduce_max_sync(kAll, __float_as_uint(x)));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void stsm4_t(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// an 8 x 8 matrix of 16-bit values over a warp, transposed: lane 4 g + c holds [g][2 c], [g][2 c + 1] before and after
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Tiles of fp16 in shared memory and in the workspace: rows of COLS values, the 16-byte piece p of row r at place p ^ swz(r), so that
// eight rows' pieces of one column (an 8 x 8 matrix of ldmatrix) lie in different banks.
template <int COLS> __device__ __forceinline__ uint32_t tile_at(int row, int piece) {
    const int sw = COLS >= 64 ? (row & 7) : ((row >> 1) & 3);
    return (uint32_t)(row * COLS * 2 + ((piece ^ sw) << 4));
}
// B fragments of n-tiles n0, n0 + 1 (8 columns each) at k-step kk from a tile [n][k]: r[0], r[1] the first tile's, r[2], r[3] the second's
template <int COLS> __device__ __forceinline__ uint32_t addr_nk(uint32_t base, int n0, int kk, int lane) {
    const int m = lane >> 3, r = lane & 7;
    return base + tile_at<COLS>(n0 * 8 + (m >> 1) * 8 + r, kk * 2 + (m & 1));
}
// the same from a tile [k][n] (with ldsm4_t)
template <int COLS> __device__ __forceinline__ uint32_t addr_kn(uint32_t base, int n0, int kk, int lane) {
    const int m = lane >> 3, r = lane & 7;
    return base + tile_at<COLS>(kk * 16 + (m & 1) * 8 + r, n0 + (m >> 1));
}
// A fragments of rows m0.. (16) at k-step kk from a tile [m][k]
template <int COLS> __device__ __forceinline__ uint32_t addr_mk(uint32_t base, int m0, int kk, int lane) {
    const int m = lane >> 3, r = lane & 7;
    return base + tile_at<COLS>(m0 + (m & 1) * 8 + r, kk * 2 + (m >> 1));
}
// A fragments from a tile [k][m] (with ldsm4_t)
template <int COLS> __device__ __forceinline__ uint32_t addr_km(uint32_t base, int m0, int kk, int lane) {
    const int m = lane >> 3, r = lane & 7;
    return base + tile_at<COLS>(kk * 16 + (m >> 1) * 8 + r, (m0 >> 3) + (m & 1));
}

// two adjacent 16 x 8 accumulator tiles as the A operand of one k-step, rows scaled by s0 (rows 0-7) and s1 (rows 8-15), in two terms
__device__ __forceinline__ void to_a(const float (&x)[4], const float (&y)[4], float s0, float s1, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    split(x[0] * s0, x[1] * s0, hi[0], lo[0]);
    split(x[2] * s1, x[3] * s1, hi[1], lo[1]);
    split(y[0] * s0, y[1] * s0, hi[2], lo[2]);
    split(y[2] * s1, y[3] * s1, hi[3], lo[3]);
}

// Tiles of 32 tokens x 16 value rows in bf16 (32 bytes a token, the two pieces of tokens 4-7 of eight exchanged): lane's address for the
// transposing ldmatrix / stmatrix of tokens 16 half .. 16 half + 15, which give and take pairs of tokens in accumulator order
__device__ __forceinline__ uint32_t tok_at(int t, int piece) { return (uint32_t)(t * 32 + ((piece ^ ((t >> 2) & 1)) << 4)); }
__device__ __forceinline__ uint32_t addr_tok(uint32_t base, int half, int lane) {
    const int m = lane >> 3, r = lane & 7;
    return base + tok_at(half * 16 + (m >> 1) * 8 + r, m & 1);
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// bulk stores from shared memory, by one lane; their reads, and the stores themselves, waited for by the same lane (others have none under way)
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_store_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// wait for a phase that has usually come: the bounded wait only if it has not
__device__ __forceinline__ void wait_phase(uint64_t* bar, uint32_t parity, const sm100::WaitCtx& w, int where) {
    if (!sm100::mbar_try_wait<false>(bar, parity)) sm100::mbar_wait(bar, parity, w, where);
}

// the first probe of a phase apart from what follows it, so that other work hides its latency
__device__ __forceinline__ bool probe_phase(uint64_t* bar, uint32_t parity) { return sm100::mbar_try_wait<false>(bar, parity); }

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(sm100::smem_u32(bar)) : "memory");
}

}  // namespace delta
}  // namespace e2ttt
