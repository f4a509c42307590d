// 8-bit checkpoints: a block of 32 values as signed bytes and a power of two.  Everything here is exact: the scale comes from the bits of the largest magnitude, a
// product with a power of two rounds nothing, and code and value meet in one addition each.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>
#include <string.h>

namespace e2ttt {
namespace pack8 {

constexpr int kBlock = 32;
constexpr uint32_t kNan = 255;  // scale byte of a block that holds a NaN or an infinity

// Scale byte e + 127 of a block whose largest magnitude has these bits: the smallest e with 127 2^e >= m 2^k, that is k - 6 up to m = 127 / 64 and k - 5 above it.  Up to
// kOrdinary, 127 2^121; what is above (and infinities and NaNs, from 0x7f800000 on) encode() sees to.
constexpr uint32_t kOrdinary = 0x7f7e0000u, kLargest = 248;
constexpr uint32_t kInfinite = 0x7f800000u;
// Logits of the recurrence count from -43 to 43 (a sigmoid is 1 there): a masked one, however far out, does not cost its block the scale, nor an infinite one its values
constexpr float kFarLogit = 43.0f;
constexpr uint32_t kFarLogitBits = 0x422c0000u;
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) { return (uint32_t)max(1, (int)((bits + 0x1ffffu) >> 23) - 6); }
__device__ __forceinline__ float scale(uint32_t byte) { return __uint_as_float(byte == kNan ? 0x7fc00000u : byte << 23); }

// two fp32 values at a time (one instruction on this architecture)
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(*reinterpret_cast<const uint64_t*>(&a)), "l"(*reinterpret_cast<const uint64_t*>(&b)), "l"(*reinterpret_cast<const uint64_t*>(&c)));
    return *reinterpret_cast<const float2*>(&r);
}
// rint(x / scale) in the low byte: 1.5 2^23 has a step of 1
__device__ __forceinline__ uint32_t code(float x, float inverse) { return __float_as_uint(fmaf(x, inverse, 12582912.0f)); }
__device__ __forceinline__ void codes2(float x, float y, float inverse, uint32_t& cx, uint32_t& cy) {
    const float2 r = fma2(make_float2(x, y), make_float2(inverse, inverse), make_float2(12582912.0f, 12582912.0f));
    cx = __float_as_uint(r.x);
    cy = __float_as_uint(r.y);
}
__device__ __forceinline__ float limited(float x) { return fminf(fmaxf(x, -0x1.fcp127f), 0x1.fcp127f); }
// low bytes of four words
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// the J-th code of a word, biased, as a number: 2^23 + 128 + code
template <int J> __device__ __forceinline__ float biased(uint32_t codes) { return __uint_as_float(__byte_perm(codes ^ 0x80808080u, 0x4b000000u, 0x7440 + J)); }
// two codes' values: (biased - (2^23 + 128)) scale, exact in one step; for scales from 2^104 on, where the product alone would be infinite (and for blocks of NaNs), in two
__device__ __forceinline__ float2 values2(float2 b, float s, bool two_steps) {
    if (two_steps) return make_float2((b.x - 8388736.0f) * s, (b.y - 8388736.0f) * s);
    const float off = -8388736.0f * s;
    return fma2(b, make_float2(s, s), make_float2(off, off));
}
__device__ __forceinline__ bool wants_two_steps(uint32_t byte) { return byte >= 231; }

// bits of the largest magnitude among neighbouring values, as they lie in memory (bits of magnitudes are in the order of their values, NaNs on top)
template <typename IO, int V> __device__ __forceinline__ uint32_t magnitude(const IO (&x)[V]) {
    uint32_t m = 0;
    if constexpr (sizeof(IO) == 2 && V % 2 == 0) {
        uint32_t w[V / 2];
        memcpy(w, x, 2 * V);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[j] & 0x7fff7fffu));
        return max(m & 0xffff0000u, m << 16);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) m = max(m, __float_as_uint((float)x[j]) & 0x7fffffffu);
        return m;
    }
}
// the same of the block of V values whose other pieces lie in the other lanes of an aligned group of 32 / V lanes; every lane of the warp calls, with in = false if it has none
template <typename IO, int V> __device__ __forceinline__ uint32_t group_magnitude(const IO (&x)[V], bool in = true) {
    uint32_t m = in ? magnitude<IO, V>(x) : 0u;
#pragma unroll
    for (int s = 1; s < kBlock / V; s <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
    return m;
}

template <int V> struct alignas(V) Codes {
    int8_t x[V];
};
// V neighbouring values as fp32
template <typename IO, int V> __device__ __forceinline__ void widen(const IO (&in)[V], float (&x)[V]) {
    if constexpr (sizeof(IO) == 2 && V % 2 == 0) {
        uint32_t w[V / 2];
        memcpy(w, in, 2 * V);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = (float)in[j];
    }
}
// Codes of V values of a block and its scale byte, from the bits of its largest magnitude.  Every lane of the warp calls: what is out of the ordinary is one branch, by a vote.
// LOGIT: the values are logits of the recurrence.
template <typename IO, int V, bool LOGIT = false> __device__ __forceinline__ Codes<V> encode(const IO (&in)[V], uint32_t bits, uint32_t& byte) {
    byte = scale_byte(bits);
    float x[V];
    widen<IO, V>(in, x);
    if (__any_sync(0xffffffffu, bits > (LOGIT ? kFarLogitBits : kOrdinary))) {
        if (LOGIT && bits <= kInfinite) {
            bits = min(bits, kFarLogitBits);
            byte = scale_byte(bits);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = fminf(fmaxf(x[j], -kFarLogit), kFarLogit);
        }
        byte = min(byte, kLargest);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = bits >= kInfinite ? 0.0f : LOGIT ? x[j] : limited(x[j]);
    }
    const float inv = __uint_as_float((254u - byte) << 23);  // 2^-e
    if (bits >= kInfinite) byte = kNan;
    Codes<V> out;
    if constexpr (V >= 4) {
        uint32_t w[V / 4];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            uint32_t c[4];
            codes2(x[4 * k], x[4 * k + 1], inv, c[0], c[1]);
            codes2(x[4 * k + 2], x[4 * k + 3], inv, c[2], c[3]);
            w[k] = bytes4(c[0], c[1], c[2], c[3]);
        }
        memcpy(&out, w, V);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out.x[j] = (int8_t)(code(x[j], inv) & 0xffu);
    }
    return out;
}
template <int V> __device__ __forceinline__ void decode(const Codes<V>& c, uint32_t byte, float (&x)[V]) {
    if constexpr (V >= 4) {
        const float s = __uint_as_float(byte << 23);  // infinite for a block of NaNs, which takes the other branch
        uint32_t w[V / 4];
        memcpy(w, &c, V);
        float2 v[V / 2];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            v[2 * k] = make_float2(biased<0>(w[k]), biased<1>(w[k]));
            v[2 * k + 1] = make_float2(biased<2>(w[k]), biased<3>(w[k]));
        }
        if (__builtin_expect(wants_two_steps(byte), 0)) {
#pragma unroll
            for (int k = 0; k < V / 2; ++k) v[k] = values2(v[k], scale(byte), true);
        } else {
#pragma unroll
            for (int k = 0; k < V / 2; ++k) v[k] = values2(v[k], s, false);
        }
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
            x[2 * k] = v[k].x;
            x[2 * k + 1] = v[k].y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = (float)c.x[j] * scale(byte);
    }
}

}  // namespace pack8
}  // namespace e2ttt
