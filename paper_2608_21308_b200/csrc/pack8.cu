// 8-bit checkpoints of activations: rows cut into blocks of 32 values, signed bytes and a power of two per block.  One pass, every byte read once and written once:
// HBM bounds it.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <string.h>

#include "../../include/e2ttt.h"
#include "api_checks.h"
#include "pack8.cuh"

namespace e2ttt {
namespace {
using namespace pack8;

__device__ __forceinline__ float ldf(float x) { return x; }
__device__ __forceinline__ float ldf(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void stf(float& y, float x) { y = x; }
__device__ __forceinline__ void stf(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

template <typename IO, int V> struct alignas(sizeof(IO) * V) Values {
    IO x[V];
};

struct PackArgs {
    int64_t rows, pieces;  // pieces: groups of V values, blocks filled up to 32
    int cols, blocks;      // blocks of a row
    const void* x;
    void* y;
    int8_t* codes;
    uint8_t* scales;
};

constexpr int kThreads = 256;

// A thread takes V neighbouring values, an aligned group of 32 / V lanes a block.
template <typename IO, int V> __global__ void __launch_bounds__(kThreads) pack8_kernel(const PackArgs a) {
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t first = (int64_t)blockIdx.x * kThreads; first < a.pieces; first += step) {
        const int64_t i = first + threadIdx.x, block = i / (kBlock / V), row = block / a.blocks;
        const int c = (int)(block - row * a.blocks) * kBlock + (int)(i % (kBlock / V)) * V;
        const bool in = i < a.pieces && c < a.cols;
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = 0.0f;
        if (in) {
            const Values<IO, V> v = *reinterpret_cast<const Values<IO, V>*>(static_cast<const IO*>(a.x) + row * a.cols + c);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = ldf(v.x[j]);
        }
        const uint32_t byte = group_scale<V>(x);
        if (!in) continue;
        *reinterpret_cast<Codes<V>*>(a.codes + row * a.cols + c) = encode<V>(x, byte);
        if (i % (kBlock / V) == 0) a.scales[block] = (uint8_t)byte;
    }
}

template <typename IO, int V> __global__ void __launch_bounds__(kThreads) unpack8_kernel(const PackArgs a) {
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.pieces; i += step) {
        const int64_t block = i / (kBlock / V), row = block / a.blocks;
        const int c = (int)(block - row * a.blocks) * kBlock + (int)(i % (kBlock / V)) * V;
        if (c >= a.cols) continue;
        float x[V];
        decode<V>(*reinterpret_cast<const Codes<V>*>(a.codes + row * a.cols + c), a.scales[block], x);
        Values<IO, V> v;
#pragma unroll
        for (int j = 0; j < V; ++j) stf(v.x[j], x[j]);
        *reinterpret_cast<Values<IO, V>*>(static_cast<IO*>(a.y) + row * a.cols + c) = v;
    }
}

template <typename IO, int V, bool PACK> int launch(PackArgs a, cudaStream_t st) {
    a.pieces = a.rows * a.blocks * (kBlock / V);
    const int64_t need = (a.pieces + kThreads - 1) / kThreads, most = 148 * 8;
    const unsigned grid = (unsigned)(need < most ? need : most);
    if (PACK) pack8_kernel<IO, V><<<grid, kThreads, 0, st>>>(a);
    else unpack8_kernel<IO, V><<<grid, kThreads, 0, st>>>(a);
    return (int)cudaGetLastError();
}

// values a thread takes: the most that the row length and the addresses allow
template <bool PACK> int dispatch(const PackArgs& a, bool f32, cudaStream_t st) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(PACK ? a.x : a.y), c = reinterpret_cast<uintptr_t>(a.codes);
    const int size = f32 ? 4 : 2;
    int v = 16 / size;
    while (v > 1 && (a.cols % v || x % (size * v) || c % v)) v >>= 1;
    if (f32) return v == 4 ? launch<float, 4, PACK>(a, st) : v == 2 ? launch<float, 2, PACK>(a, st) : launch<float, 1, PACK>(a, st);
    return v == 8   ? launch<__nv_bfloat16, 8, PACK>(a, st)
           : v == 4 ? launch<__nv_bfloat16, 4, PACK>(a, st)
           : v == 2 ? launch<__nv_bfloat16, 2, PACK>(a, st)
                    : launch<__nv_bfloat16, 1, PACK>(a, st);
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
    const PackArgs a{p->rows, 0, p->cols, (int)blocks, x, y, codes, scales};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool f32 = p->io_dtype == E2TTT_F32;
    return (x ? dispatch<true>(a, f32, st) : dispatch<false>(a, f32, st)) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
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
