// 8-bit checkpoints of activations: rows cut into blocks of 32 values, signed bytes and a power of two per block.  One pass, every byte read once and written once:
// HBM bounds it.  A lane takes 16 bytes of x at a time (less where rows or addresses do not allow it) and an aligned group of lanes a block, whose largest magnitude takes two or three
// shuffles; four such pieces are under way per lane.  16384 x 2048 in bf16: 19 us (102 MB, 5.4 TB/s), 21 to read back; rows of 2047, a value
// at a time, 107 and 80 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <string.h>

#include "../../include/e2ttt.h"
#include "api_checks.h"
#include "pack8.cuh"

namespace e2ttt {
namespace {
using namespace pack8;

__device__ __forceinline__ void stf(float& y, float x) { y = x; }
__device__ __forceinline__ void stf(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

template <typename IO, int V> struct alignas(sizeof(IO) * V) Values {
    IO x[V];
};

struct PackArgs {
    int64_t pieces;  // groups of V values, every row's last block filled up to 32
    int cols, blocks;  // blocks of a row
    const void* x;
    void* y;
    int8_t* codes;
    uint8_t* scales;
};

constexpr int kThreads = 256, kDeep = 4;

// Where a piece lies.  FLAT: rows are whole blocks, so that they follow one another without a gap.
template <int V, bool FLAT> struct Place {
    int64_t block, at;
    bool in;
    __device__ __forceinline__ Place(const PackArgs& a, int64_t i) {
        block = i / (kBlock / V);
        in = i < a.pieces;
        if (FLAT) {
            at = i * V;
        } else {
            const int64_t row = a.pieces >> 31 ? block / a.blocks : (int64_t)((uint32_t)block / (uint32_t)a.blocks);
            const int c = (int)(block - row * a.blocks) * kBlock + (int)(i % (kBlock / V)) * V;
            at = row * a.cols + c;
            in = in && c < a.cols;
        }
    }
};

template <typename IO, int V, bool FLAT> __global__ void __launch_bounds__(kThreads) pack8_kernel(const PackArgs a) {
    const int64_t first = (int64_t)blockIdx.x * (kThreads * kDeep) + threadIdx.x;
    Values<IO, V> v[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
        const Place<V, FLAT> p(a, first + k * kThreads);
        if (p.in) v[k] = *reinterpret_cast<const Values<IO, V>*>(static_cast<const IO*>(a.x) + p.at);
    }
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
        const Place<V, FLAT> p(a, first + k * kThreads);
        uint32_t byte;
        const Codes<V> code = encode<IO, V>(v[k].x, group_magnitude<IO, V>(v[k].x, p.in), byte);
        if (!p.in) continue;
        *reinterpret_cast<Codes<V>*>(a.codes + p.at) = code;
        if (threadIdx.x % (kBlock / V) == 0) a.scales[p.block] = (uint8_t)byte;
    }
}

template <typename IO, int V, bool FLAT> __global__ void __launch_bounds__(kThreads) unpack8_kernel(const PackArgs a) {
    const int64_t first = (int64_t)blockIdx.x * (kThreads * kDeep) + threadIdx.x;
    Codes<V> c[kDeep];
    uint32_t byte[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
        const Place<V, FLAT> p(a, first + k * kThreads);
        if (!p.in) continue;
        c[k] = *reinterpret_cast<const Codes<V>*>(a.codes + p.at);
        byte[k] = a.scales[p.block];
    }
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
        const Place<V, FLAT> p(a, first + k * kThreads);
        if (!p.in) continue;
        float x[V];
        decode<V>(c[k], byte[k], x);
        Values<IO, V> v;
#pragma unroll
        for (int j = 0; j < V; ++j) stf(v.x[j], x[j]);
        *reinterpret_cast<Values<IO, V>*>(static_cast<IO*>(a.y) + p.at) = v;
    }
}

template <typename IO, int V, bool PACK, bool FLAT> int launch(const PackArgs& a, cudaStream_t st) {
    const unsigned grid = (unsigned)((a.pieces + kThreads * kDeep - 1) / (kThreads * kDeep));
    if (PACK) pack8_kernel<IO, V, FLAT><<<grid, kThreads, 0, st>>>(a);
    else unpack8_kernel<IO, V, FLAT><<<grid, kThreads, 0, st>>>(a);
    return (int)cudaGetLastError();
}
template <typename IO, int V, bool PACK> int launch(PackArgs a, int64_t rows, cudaStream_t st) {
    a.pieces = rows * a.blocks * (kBlock / V);
    return a.cols % kBlock == 0 ? launch<IO, V, PACK, true>(a, st) : launch<IO, V, PACK, false>(a, st);
}

// values a thread takes: the most that the row length and the addresses allow
template <bool PACK> int dispatch(const PackArgs& a, int64_t rows, bool f32, cudaStream_t st) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(PACK ? a.x : a.y), c = reinterpret_cast<uintptr_t>(a.codes);
    const int size = f32 ? 4 : 2;
    int v = 16 / size;
    while (v > 1 && (a.cols % v || x % (size * v) || c % v)) v >>= 1;
    if (f32) return v == 4 ? launch<float, 4, PACK>(a, rows, st) : v == 2 ? launch<float, 2, PACK>(a, rows, st) : launch<float, 1, PACK>(a, rows, st);
    return v == 8   ? launch<__nv_bfloat16, 8, PACK>(a, rows, st)
           : v == 4 ? launch<__nv_bfloat16, 4, PACK>(a, rows, st)
           : v == 2 ? launch<__nv_bfloat16, 2, PACK>(a, rows, st)
                    : launch<__nv_bfloat16, 1, PACK>(a, rows, st);
}

int run(const e2ttt_pack_params* p, const void* x, void* y, int8_t* codes, uint8_t* scales, void* stream) {
    if (!p) return E2TTT_ERR_NULL;
    if (p->io_dtype != E2TTT_F32 && p->io_dtype != E2TTT_BF16) return E2TTT_ERR_DTYPE;
    if (p->rows <= 0 || p->cols <= 0 || p->rows > (int64_t)1 << 40 || p->cols > (1 << 30)) return E2TTT_ERR_SHAPE;
    const int64_t blocks = ((int64_t)p->cols + kBlock - 1) / kBlock;
    if (p->rows > ((int64_t)1 << 40) / (blocks * kBlock)) return E2TTT_ERR_SHAPE;
    const void* data = x ? x : y;
    if (!data || !codes || !scales) return E2TTT_ERR_NULL;
    if (!aligned(data, p->io_dtype == E2TTT_F32 ? 4 : 2)) return E2TTT_ERR_ALIGN;
    const int rc = check_device();
    if (rc) return rc;
    const PackArgs a{0, p->cols, (int)blocks, x, y, codes, scales};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool f32 = p->io_dtype == E2TTT_F32;
    return (x ? dispatch<true>(a, p->rows, f32, st) : dispatch<false>(a, p->rows, f32, st)) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

}  // namespace
}  // namespace e2ttt

extern "C" {

int e2ttt_pack8(const e2ttt_pack_params* p, const void* x, int8_t* codes, uint8_t* scales, void* stream) {
    return e2ttt::run(p, x, nullptr, codes, scales, stream);
}
int e2ttt_unpack8(const e2ttt_pack_params* p, const int8_t* codes, const uint8_t* scales, void* x, void* stream) {
    return e2ttt::run(p, nullptr, x, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), stream);
}

}  // extern "C"
