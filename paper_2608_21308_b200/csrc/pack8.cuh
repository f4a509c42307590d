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

// Scale byte e + 127 of a block whose largest magnitude has these bits: the smallest e with 127 2^e >= m 2^k, that is k - 6 up to m = 127 / 64 and k - 5 above it.
// An infinity or a NaN has bits from 0x7f800000 on (a NaN must arrive as its bits: compare as integers, not by fmaxf).
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
    const int e = (int)((bits + 0x1ffffu) >> 23) - 6;
    return bits >= 0x7f800000u ? kNan : (uint32_t)max(1, min(248, e));
}
// 2^-e; 0 for a block that is not finite
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float(byte == kNan ? 0u : (254u - byte) << 23); }
__device__ __forceinline__ float scale(uint32_t byte) { return __uint_as_float(byte == kNan ? 0x7fc00000u : byte << 23); }

// rint(x / scale) in the low byte: 1.5 2^23 has a step of 1
__device__ __forceinline__ uint32_t code(float x, float inverse) { return __float_as_uint(fmaf(x, inverse, 12582912.0f)); }
constexpr uint32_t kLargest = 248;  // scale byte of 2^121: the only one with values above 127 of its units
__device__ __forceinline__ float limited(float x) { return fminf(fmaxf(x, -0x1.fcp127f), 0x1.fcp127f); }
// low bytes of four words
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// the J-th code of a word, as a number: 2^23 + (code + 128), less 2^23 + 128
template <int J> __device__ __forceinline__ float number(uint32_t codes) {
    return __uint_as_float(__byte_perm(codes ^ 0x80808080u, 0x4b000000u, 0x7440 + J)) - 8388736.0f;
}

// bits of the largest magnitude among neighbouring values, as they lie in memory (bits of magnitudes are in the order of their values, NaNs on top)
template <typename IO, int V> __device__ __forceinline__ uint32_t magnitude(const IO (&x)[V]) {
    uint32_t m = 0;
    if constexpr (sizeof(IO) == 2 && V % 2 == 0) {
        uint32_t w[V / 2];
        memcpy(w, x, 2 * V);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) m = __vmaxu2(m, w[j] & 0x7fff7fffu);
        return max(m & 0xffff0000u, m << 16);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) m = max(m, __float_as_uint((float)x[j]) & 0x7fffffffu);
        return m;
    }
}
// the scale byte of V values whose block's other pieces lie in the other lanes of an aligned group of 32 / V lanes; every lane of the warp calls
template <typename IO, int V> __device__ __forceinline__ uint32_t group_scale(const IO (&x)[V]) {
    uint32_t m = magnitude<IO, V>(x);
#pragma unroll
    for (int s = 1; s < kBlock / V; s <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
    return scale_byte(m);
}

template <int V> struct alignas(V) Codes {
    int8_t x[V];
};
template <typename IO, int V> __device__ __forceinline__ Codes<V> encode(const IO (&in)[V], uint32_t byte) {
    const float inv = inverse_scale(byte);
    float x[V];
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = (float)in[j];
    if (byte >= kLargest) {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = byte == kNan ? 0.0f : limited(x[j]);
    }
    Codes<V> out;
    if constexpr (V >= 4) {
        uint32_t w[V / 4];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) w[k] = bytes4(code(x[4 * k], inv), code(x[4 * k + 1], inv), code(x[4 * k + 2], inv), code(x[4 * k + 3], inv));
        memcpy(&out, w, V);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out.x[j] = (int8_t)(code(x[j], inv) & 0xffu);
    }
    return out;
}
template <int V> __device__ __forceinline__ void decode(const Codes<V>& c, uint32_t byte, float (&x)[V]) {
    const float s = scale(byte);
    if constexpr (V >= 4) {
        uint32_t w[V / 4];
        memcpy(w, &c, V);
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            x[4 * k] = number<0>(w[k]) * s;
            x[4 * k + 1] = number<1>(w[k]) * s;
            x[4 * k + 2] = number<2>(w[k]) * s;
            x[4 * k + 3] = number<3>(w[k]) * s;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = (float)c.x[j] * s;
    }
}

}  // namespace pack8
}  // namespace e2ttt
