// Block join, forward and reverse pass.  Per token, o [B,H,L,d] by heads, everything else [B,L,H d]:
//   y = o / rms(o per head) w_post,   z = gate(a) y,   x_out = x + res_scale z,   n = x_out / rms(x_out) w_pre.
// Every tensor is read once and written once: HBM bounds both passes.  A CTA takes a token at a time, a thread V neighbouring values of
// it (16 bytes where widths and addresses allow); a head's sum is a few shuffles where a head's pieces fill an aligned part of a
// warp, else it goes through shared memory.
// Reverse pass, with r = gate(a) y0, y0 = o / rms(o):  d x = d x_out + (adjoint of the second norm),  d w_post = res_scale sum_tokens(dx r),
// d res_scale = w_post sum_tokens(dx r): one column sum serves both, a second one is d w_pre.  A CTA keeps its tokens' column sums in
// registers; the CTAs' sums are added by a second launch in a fixed order, so that results repeat bit for bit.
// 16384 tokens of 2048 in bf16 with a gate and both norms: 64 us forward (336 MB, 5.2 TB/s), 131 us in reverse (537 MB, 4.1 TB/s) and 6 us for the column
// sums; 8000 tokens of 768 in fp32, sigmoid gate: 31, 58 and 7 us.  What is above the bytes' time is
// issue with heads that fit a warp (the gate's special functions, bf16 conversions, sums), and the barriers of the sums through shared memory with wider ones.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <initializer_list>

#include "../../include/e2ttt.h"
#include "api_checks.h"
#include "join.h"

namespace e2ttt {
namespace {

constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float ldf(float x) { return x; }
__device__ __forceinline__ float ldf(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void stf(float& y, float x) { y = x; }
__device__ __forceinline__ void stf(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

template <typename IO, int V> struct alignas(sizeof(IO) * V) Piece {
    IO x[V];
};

// 1 / (1 + exp(-a)).  The hardware's reciprocal is off by one step of fp32 (2^-23), which a division would halve.  With bf16 I/O what the gate enters is
// rounded to 2^-9 right after, and the hardware's exponential (2^-22, and that of its argument) serves as well.  a -> -inf: the exponential is inf, the result 0.
template <typename IO> __device__ __forceinline__ float sigmoid(float a) {
    float e, r;
    if (sizeof(IO) == 4) e = expf(-a);
    else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(a * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

// The smaller of sig = sigmoid(a) and 1 - sig: e / (1 + e), e = exp(-|a|).  The reverse pass needs both, and 1 - sig as a difference would lose what an open gate's
// derivative is made of (all of it from a = 17 on).
template <typename IO> __device__ __forceinline__ float smaller_part(float a) {
    float e, r;
    if (sizeof(IO) == 4) e = expf(-fabsf(a));
    else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(a) * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return e * r;
}

// Where a token's rows of o start: its batch and position, moved on by the grid's size without a division.
struct Place {
    int64_t base;  // first piece of (batch, head 0, position)
    int l;
    __device__ __forceinline__ Place(const JoinArgs& a, int64_t tok, int G) {
        const int64_t b = tok / a.L;
        l = (int)(tok - b * a.L);
        base = (b * a.H * a.L + l) * G;
    }
};
struct Stride {
    int64_t step, wrap;  // pieces to move on, and more when the position wraps into the next batch row
    int dl, L;
    __device__ __forceinline__ Stride(const JoinArgs& a, int64_t by, int G) {
        const int64_t db = by / a.L;
        L = a.L;
        dl = (int)(by - db * a.L);
        step = (db * a.H * a.L + dl) * G;
        wrap = (int64_t)(a.H - 1) * a.L * G;
    }
    __device__ __forceinline__ void move(Place& p) const {
        p.base += step;
        p.l += dl;
        if (p.l >= L) { p.l -= L; p.base += wrap; }
    }
};

// Sums over a token's heads and over the token.  `cols` pieces of V values; a head has G of them.
struct Sums {
    float *part, *head, *row;  // shared memory: [cols], [H], [2][2][16]
    int cols, G, H, T, flip;
    bool lanes;                // a head is an aligned group of G lanes
};

// v[i]: sum over piece i of the thread -> sum over the piece's head
template <int NC> __device__ __forceinline__ void head_sums(Sums& s, float (&v)[NC]) {
    const int tid = threadIdx.x;
    if (s.lanes) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
            for (int x = 1; x < s.G; x <<= 1) v[i] += __shfl_xor_sync(kAll, v[i], x);
        return;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (tid + i * s.T < s.cols) s.part[tid + i * s.T] = v[i];
    __syncthreads();
    for (int h = tid >> 5; h < s.H; h += s.T >> 5) {
        float y = 0.0f;
        for (int j = tid & 31; j < s.G; j += 32) y += s.part[h * s.G + j];
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) y += __shfl_xor_sync(kAll, y, x);
        if ((tid & 31) == 0) s.head[h] = y;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (tid + i * s.T < s.cols) v[i] = s.head[(tid + i * s.T) / s.G];
}

// sums of u[0] (and u[1]) over the CTA's threads, in a fixed order; two buffers in turn, so that one barrier is enough.  A warp's lanes 0-15 read the
// warps' first sums, lanes 16-31 the second ones.
template <int N> __device__ __forceinline__ void row_sums(Sums& s, float (&u)[N]) {
#pragma unroll
    for (int x = 16; x > 0; x >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) u[k] += __shfl_xor_sync(kAll, u[k], x);
    const int warps = s.T >> 5, lane = threadIdx.x & 31;
    if (warps == 1) return;
    float* b = s.row + s.flip * 32;
    s.flip ^= 1;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) b[16 * k + (threadIdx.x >> 5)] = u[k];
    }
    __syncthreads();
    float y = (lane & 15) < warps ? b[N == 1 ? lane & 15 : lane] : 0.0f;
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) y += __shfl_xor_sync(kAll, y, x);
    u[0] = N == 1 ? y : __shfl_sync(kAll, y, 0);
    if (N == 2) u[N - 1] = __shfl_sync(kAll, y, 16);
}

__device__ __forceinline__ Sums make_sums(char* smem, int cols, int G, int H) {
    Sums s;
    s.row = reinterpret_cast<float*>(smem);
    s.part = s.row + 64;
    s.head = s.part + cols;
    s.cols = cols; s.G = G; s.H = H; s.T = blockDim.x; s.flip = 0;
    s.lanes = G <= 32 && (G & (G - 1)) == 0;
    return s;
}

// A thread's pieces of the tokens to come wait in shared memory, `depth` tokens deep: cp.async needs no registers for what is in flight, and as
// every thread reads back only what it copied itself, no barrier either.
template <int BYTES> __device__ __forceinline__ void copy_piece(void* dst, const void* src) {
    if constexpr (BYTES >= 4) {
        const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
        if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(BYTES) : "memory");
    } else {
        *reinterpret_cast<uint16_t*>(dst) = *reinterpret_cast<const uint16_t*>(src);
    }
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait(int pending) {  // until at most that many groups are under way
    switch (pending) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}
template <int V> struct alignas(V >= 4 ? 16 : 4 * V) Weights {
    float x[V];
};
template <int V> __device__ __forceinline__ Weights<V> weights(const float* w, int c) { return reinterpret_cast<const Weights<V>*>(w)[c]; }

// Whether a thread of the forward keeps its weights in registers from token to token (three CTAs of 256 threads on an SM instead of four).  16384 tokens
// of 2048 in bf16: 65 us with them, 72 without; fp32, whose threads take two pieces of four, 8000 tokens of 768: 41 and 35.
template <int V, int TMAX> constexpr bool kept() { return V == 8 && TMAX == 256; }

template <typename IO, int V, int NC, int TMAX>
__global__ void __launch_bounds__(TMAX, kept<V, TMAX>() ? 3 : 1024 / TMAX) join_fwd_kernel(const JoinArgs a, const int depth) {
    extern __shared__ __align__(16) char smem[];
    using P = Piece<IO, V>;
    const int D = a.H * a.d, cols = D / V, T = blockDim.x, tid = threadIdx.x;
    P* ring = reinterpret_cast<P*>(smem) + tid;  // [depth][3][NC][T]
    Sums sums = make_sums(smem + (size_t)depth * 3 * NC * T * sizeof(P), cols, a.d / V, a.H);
    const int64_t tokens = (int64_t)a.B * a.L;
    int64_t own[NC];  // a piece of o within its token: head and place in the head
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * T, h = c / sums.G;
        own[i] = (int64_t)h * a.L * sums.G + (c - h * sums.G);
    }
    const float per_d = 1.0f / a.d, per_D = 1.0f / D;
    const bool silu = a.gate == E2TTT_GATE_SILU;
    Place ahead(a, blockIdx.x, sums.G);
    const Stride stride(a, gridDim.x, sums.G);
    auto load = [&](int64_t tok, int slot) {
        if (tok < tokens) {
            P* r = ring + slot * 3 * NC * T;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = tid + i * T;
                if (c >= cols) continue;
                copy_piece<sizeof(P)>(r + i * T, reinterpret_cast<const P*>(a.o) + ahead.base + own[i]);
                copy_piece<sizeof(P)>(r + (NC + i) * T, reinterpret_cast<const P*>(a.x) + tok * cols + c);
                if (a.a) copy_piece<sizeof(P)>(r + (2 * NC + i) * T, reinterpret_cast<const P*>(a.a) + tok * cols + c);
            }
        }
        stride.move(ahead);
        copy_commit();
    };
    Weights<V> wrs[NC], wps[NC], wns[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * T;
        if (!kept<V, TMAX>() || c >= cols) continue;
        wrs[i] = weights<V>(a.res_scale, c);
        wps[i] = weights<V>(a.w_post, c);
        if (a.w_pre) wns[i] = weights<V>(a.w_pre, c);
    }
    int64_t tok = blockIdx.x;
    for (int i = 0; i + 1 < depth; ++i) load(tok + i * (int64_t)gridDim.x, i);
    int slot = 0;
    for (; tok < tokens; tok += gridDim.x) {
        load(tok + (depth - 1) * (int64_t)gridDim.x, slot == 0 ? depth - 1 : slot - 1);
        copy_wait(depth - 1);
        const P* r = ring + slot * 3 * NC * T;
        slot = slot + 1 == depth ? 0 : slot + 1;
        float y[NC][V], hs[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            hs[i] = 0.0f;
            if (tid + i * T >= cols) continue;
            const P po = r[i * T];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[i][j] = ldf(po.x[j]);
                hs[i] = fmaf(y[i][j], y[i][j], hs[i]);
            }
        }
        head_sums<NC>(sums, hs);
        float sum[1] = {0.0f};  // of x_out^2
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + i * T;
            if (c >= cols) continue;
            const float inv = rsqrtf(fmaf(hs[i], per_d, a.post_eps));
            const P px = r[(NC + i) * T], pa = r[(2 * NC + i) * T];
            const Weights<V> wr = kept<V, TMAX>() ? wrs[i] : weights<V>(a.res_scale, c), wp = kept<V, TMAX>() ? wps[i] : weights<V>(a.w_post, c);
            if (a.a) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float av = ldf(pa.x[j]), sig = sigmoid<IO>(av);
                    y[i][j] *= silu ? av * sig : sig;
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[i][j] = fmaf(wr.x[j] * inv, y[i][j] * wp.x[j], ldf(px.x[j]));
                sum[0] = fmaf(y[i][j], y[i][j], sum[0]);
            }
        }
        if (a.w_pre) row_sums<1>(sums, sum);
        const float m = rsqrtf(fmaf(sum[0], per_D, a.pre_eps));
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + i * T;
            if (c >= cols) continue;
            P xo, nn;
#pragma unroll
            for (int j = 0; j < V; ++j) stf(xo.x[j], y[i][j]);
            reinterpret_cast<P*>(a.x_out)[tok * cols + c] = xo;
            if (a.w_pre) {
                const Weights<V> w = kept<V, TMAX>() ? wns[i] : weights<V>(a.w_pre, c);
#pragma unroll
                for (int j = 0; j < V; ++j) stf(nn.x[j], y[i][j] * m * w.x[j]);
                reinterpret_cast<P*>(a.n_out)[tok * cols + c] = nn;
            }
        }
    }
}

template <typename IO, int V, int NC, int TMAX>
__global__ void __launch_bounds__(TMAX, 512 / TMAX) join_bwd_kernel(const JoinBwdArgs ba, const int depth) {
    extern __shared__ __align__(16) char smem[];
    using P = Piece<IO, V>;
    constexpr bool KEPT = TMAX == 256;
    const JoinArgs& a = ba.f;
    const int D = a.H * a.d, cols = D / V, T = blockDim.x, tid = threadIdx.x;
    P* ring = reinterpret_cast<P*>(smem) + tid;  // [depth][5][NC][T]
    Sums sums = make_sums(smem + (size_t)depth * 5 * NC * T * sizeof(P), cols, a.d / V, a.H);
    const int64_t tokens = (int64_t)a.B * a.L;
    int64_t own[NC];  // a piece of o within its token: head and place in the head
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * T, h = c / sums.G;
        own[i] = (int64_t)h * a.L * sums.G + (c - h * sums.G);
    }
    const float per_d = 1.0f / a.d, per_D = 1.0f / D;
    const bool silu = a.gate == E2TTT_GATE_SILU;
    Place ahead(a, blockIdx.x, sums.G);
    const Stride stride(a, gridDim.x, sums.G);
    auto load = [&](int64_t tok, int slot) {
        if (tok < tokens) {
            P* r = ring + slot * 5 * NC * T;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = tid + i * T;
                if (c >= cols) continue;
                copy_piece<sizeof(P)>(r + i * T, reinterpret_cast<const P*>(a.o) + ahead.base + own[i]);
                copy_piece<sizeof(P)>(r + (NC + i) * T, reinterpret_cast<const P*>(a.x) + tok * cols + c);
                if (a.a) copy_piece<sizeof(P)>(r + (2 * NC + i) * T, reinterpret_cast<const P*>(a.a) + tok * cols + c);
                copy_piece<sizeof(P)>(r + (3 * NC + i) * T, reinterpret_cast<const P*>(ba.d_x_out) + tok * cols + c);
                if (a.w_pre) copy_piece<sizeof(P)>(r + (4 * NC + i) * T, reinterpret_cast<const P*>(ba.d_n) + tok * cols + c);
            }
        }
        stride.move(ahead);
        copy_commit();
    };
    Place here = ahead;
    float R[NC][V], W[NC][V];  // column sums: dx gate y0, and dn x_out / rms
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) R[i][j] = W[i][j] = 0.0f;
    Weights<V> wrs[NC], wps[NC], wns[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * T;
        if (!KEPT || c >= cols) continue;
        wrs[i] = weights<V>(a.res_scale, c);
        wps[i] = weights<V>(a.w_post, c);
        if (a.w_pre) wns[i] = weights<V>(a.w_pre, c);
    }
    int64_t tok = blockIdx.x;
    for (int i = 0; i + 1 < depth; ++i) load(tok + i * (int64_t)gridDim.x, i);
    int slot = 0;
    for (; tok < tokens; tok += gridDim.x) {
        load(tok + (depth - 1) * (int64_t)gridDim.x, slot == 0 ? depth - 1 : slot - 1);
        copy_wait(depth - 1);
        const P* r = ring + slot * 5 * NC * T;
        slot = slot + 1 == depth ? 0 : slot + 1;
        float y[NC][V], xo[NC][V], sg[NC][V], hs[NC], inv[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            hs[i] = 0.0f;
            if (tid + i * T >= cols) continue;
            const P po = r[i * T];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[i][j] = ldf(po.x[j]);
                hs[i] = fmaf(y[i][j], y[i][j], hs[i]);
            }
        }
        head_sums<NC>(sums, hs);
        float sum[2] = {0.0f, 0.0f};  // of x_out^2 and of dn w x_out
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + i * T;
            if (c >= cols) continue;
            inv[i] = rsqrtf(fmaf(hs[i], per_d, a.post_eps));
            const P px = r[(NC + i) * T], pa = r[(2 * NC + i) * T], pn = r[(4 * NC + i) * T];
            const Weights<V> wr = KEPT ? wrs[i] : weights<V>(a.res_scale, c), wp = KEPT ? wps[i] : weights<V>(a.w_post, c);
#pragma unroll
            for (int j = 0; j < V; ++j) xo[i][j] = 1.0f;
            if (a.a) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float av = ldf(pa.x[j]), w = smaller_part<IO>(av), sig = av > 0.0f ? 1.0f - w : w;
                    if (KEPT) sg[i][j] = w;
                    xo[i][j] = silu ? av * sig : sig;
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[i][j] *= inv[i];
                xo[i][j] = fmaf(wr.x[j] * xo[i][j], y[i][j] * wp.x[j], ldf(px.x[j]));
                sum[0] = fmaf(xo[i][j], xo[i][j], sum[0]);
            }
            if (a.w_pre) {
                const Weights<V> w = KEPT ? wns[i] : weights<V>(a.w_pre, c);
#pragma unroll
                for (int j = 0; j < V; ++j) sum[1] = fmaf(ldf(pn.x[j]) * w.x[j], xo[i][j], sum[1]);
            }
        }
        float m = 0.0f, mean = 0.0f;
        if (a.w_pre) {
            row_sums<2>(sums, sum);
            m = rsqrtf(fmaf(sum[0], per_D, a.pre_eps));
            mean = sum[1] * m * per_D;
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + i * T;
            hs[i] = 0.0f;
            if (c >= cols) continue;
            const P pa = r[(2 * NC + i) * T], pd = r[(3 * NC + i) * T], pn = r[(4 * NC + i) * T];
            float dx[V];
#pragma unroll
            for (int j = 0; j < V; ++j) dx[j] = ldf(pd.x[j]);
            if (a.w_pre) {
                const Weights<V> w = KEPT ? wns[i] : weights<V>(a.w_pre, c);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float dn = ldf(pn.x[j]), h = xo[i][j] * m;
                    W[i][j] = fmaf(dn, h, W[i][j]);
                    dx[j] = fmaf(m, fmaf(-h, mean, dn * w.x[j]), dx[j]);
                }
            }
            P dx_p;
            const Weights<V> wr = KEPT ? wrs[i] : weights<V>(a.res_scale, c), wp = KEPT ? wps[i] : weights<V>(a.w_post, c);
#pragma unroll
            for (int j = 0; j < V; ++j) stf(dx_p.x[j], dx[j]);
            reinterpret_cast<P*>(ba.d_x)[tok * cols + c] = dx_p;
            if (a.a) {
                P da_p;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float av = ldf(pa.x[j]), w = KEPT ? sg[i][j] : smaller_part<IO>(av);
                    const float sig = av > 0.0f ? 1.0f - w : w, rest = av > 0.0f ? w : 1.0f - w, dev = silu ? fmaf(av, rest, 1.0f) : rest;
                    stf(da_p.x[j], dx[j] * wr.x[j] * wp.x[j] * y[i][j] * (sig * dev));
                    dx[j] *= silu ? av * sig : sig;
                }
                reinterpret_cast<P*>(ba.d_a)[tok * cols + c] = da_p;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                R[i][j] = fmaf(dx[j], y[i][j], R[i][j]);
                xo[i][j] = dx[j] * wr.x[j] * wp.x[j];  // adjoint of y0
                hs[i] = fmaf(xo[i][j], y[i][j], hs[i]);
            }
        }
        head_sums<NC>(sums, hs);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + i * T;
            if (c >= cols) continue;
            const float mh = hs[i] * per_d;
            P do_p;
#pragma unroll
            for (int j = 0; j < V; ++j) stf(do_p.x[j], inv[i] * fmaf(-y[i][j], mh, xo[i][j]));
            reinterpret_cast<P*>(ba.d_o)[here.base + own[i]] = do_p;
        }
        stride.move(here);
    }
    float* part = ba.part + (size_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * T;
        if (c >= cols) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            part[c * V + j] = R[i][j];
            if (a.w_pre) part[D + c * V + j] = W[i][j];
        }
    }
}

// Column sums over the CTAs' partial sums: 8 columns (32 bytes of a row) by 128 row groups a CTA, so that many SMs have a part of the few MB.  Both sums of a
// column are added in an order that depends on the number of rows alone.
constexpr int kSumCols = 8;
__global__ void __launch_bounds__(1024) join_sum_kernel(const JoinBwdArgs ba, const int rows) {
    __shared__ float red[2][kSumCols][33];
    const JoinArgs& a = ba.f;
    const int D = a.H * a.d, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = lane & 7, c = blockIdx.x * kSumCols + col;
    float r = 0.0f, w = 0.0f;
    if (c < D) {
#pragma unroll 4
        for (int i = threadIdx.x >> 3; i < rows; i += 128) {
            r += ba.part[(size_t)i * 2 * D + c];
            if (a.w_pre) w += ba.part[(size_t)i * 2 * D + D + c];
        }
    }
#pragma unroll
    for (int x = 8; x <= 16; x <<= 1) {
        r += __shfl_xor_sync(kAll, r, x);
        w += __shfl_xor_sync(kAll, w, x);
    }
    if (lane < kSumCols) { red[0][lane][warp] = r; red[1][lane][warp] = w; }
    __syncthreads();
    if (warp >= kSumCols) return;
    r = red[0][warp][lane];
    w = red[1][warp][lane];
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) {
        r += __shfl_xor_sync(kAll, r, x);
        w += __shfl_xor_sync(kAll, w, x);
    }
    const int out = blockIdx.x * kSumCols + warp;
    if (lane != 0 || out >= D) return;
    ba.d_w_post[out] = r * a.res_scale[out];
    ba.d_res_scale[out] = r * a.w_post[out];
    if (a.w_pre) ba.d_w_pre[out] = w;
}

// values per piece: the widest that divides a head and that all addresses allow
int piece_of(const JoinArgs& a, std::initializer_list<const void*> ptrs) {
    const int size = a.f32 ? 4 : 2;
    int v = 16 / size;
    uintptr_t all = 0, w = 0;
    for (const void* p : ptrs) all |= reinterpret_cast<uintptr_t>(p);
    for (const void* p : {a.w_post, a.res_scale, a.w_pre}) w |= reinterpret_cast<uintptr_t>(p);
    while (v > 1 && (a.d % v || all % (size * v) || w % (v >= 4 ? 16 : 4 * v))) v >>= 1;
    return v;
}

struct Shape {
    int threads, depth, smem;
};
// tensors: how many are read per token; room: shared memory that a CTA may take for its ring where more than one token is to be under way
Shape shape_of(const JoinArgs& a, int V, int NC, int tensors, int room) {
    const int cols = a.H * a.d / V, t = ((cols + NC - 1) / NC + 31) / 32 * 32;
    const int stage = tensors * NC * t * V * (a.f32 ? 4 : 2), G = a.d / V;
    const bool lanes = G <= 32 && (G & (G - 1)) == 0;
    int depth = room / stage;
    depth = depth > 4 ? 4 : (depth < 1 ? 1 : depth);
    return {t, depth, depth * stage + (64 + (lanes ? 0 : cols + a.H)) * 4};
}

template <typename IO, int V, int NC, int TMAX> int launch_fwd(const JoinArgs& a, const Shape& s, cudaStream_t st) {
    auto kernel = join_fwd_kernel<IO, V, NC, TMAX>;
    cudaError_t e = allow_shared_memory<join_fwd_kernel<IO, V, NC, TMAX>>();
    if (e != cudaSuccess) return (int)e;
    constexpr int threads = kept<V, TMAX>() ? 768 : 1024;  // on an SM
    const int64_t tokens = (int64_t)a.B * a.L, most = 148 * (threads / s.threads > 16 ? 16 : threads / s.threads);
    kernel<<<(unsigned)(tokens < most ? tokens : most), s.threads, s.smem, st>>>(a, s.depth);
    return (int)cudaGetLastError();
}
template <typename IO, int V, int NC, int TMAX> int launch_bwd(const JoinBwdArgs& b, const Shape& s, cudaStream_t st) {
    auto kernel = join_bwd_kernel<IO, V, NC, TMAX>;
    cudaError_t e = allow_shared_memory<join_bwd_kernel<IO, V, NC, TMAX>>();
    if (e != cudaSuccess) return (int)e;
    const int grid = join_bwd_grid((int64_t)b.f.B * b.f.L, b.f.H * b.f.d);
    kernel<<<grid, s.threads, s.smem, st>>>(b, s.depth);
    e = cudaGetLastError();
    if (e != cudaSuccess) return (int)e;
    join_sum_kernel<<<(b.f.H * b.f.d + kSumCols - 1) / kSumCols, 1024, 0, st>>>(b, grid);
    return (int)cudaGetLastError();
}

template <typename IO, int V, int NC> int sized(const JoinArgs& a, cudaStream_t st) {
    const Shape s = shape_of(a, V, NC, 3, 56 * 1024);
    if constexpr (V * NC == 8)
        if (s.threads <= 256) return launch_fwd<IO, V, NC, 256>(a, s, st);
    return launch_fwd<IO, V, NC, 512>(a, s, st);
}
template <typename IO, int V, int NC> int sized(const JoinBwdArgs& b, cudaStream_t st) {
    const Shape s = shape_of(b.f, V, NC, 5, 110 * 1024);
    if constexpr (V * NC == 8)
        if (s.threads <= 256) return launch_bwd<IO, V, NC, 256>(b, s, st);
    return launch_bwd<IO, V, NC, 512>(b, s, st);
}
// 8 values a thread up to 4096 columns (512 threads), 16 above
template <typename IO, typename Args> int dispatch(const Args& args, int v, bool wide, cudaStream_t st) {
    if constexpr (sizeof(IO) == 2)
        if (v == 8) return wide ? sized<IO, 8, 2>(args, st) : sized<IO, 8, 1>(args, st);
    if (v == 4) return wide ? sized<IO, 4, 4>(args, st) : sized<IO, 4, 2>(args, st);
    if (v == 2) return wide ? sized<IO, 2, 8>(args, st) : sized<IO, 2, 4>(args, st);
    return wide ? sized<IO, 1, 16>(args, st) : sized<IO, 1, 8>(args, st);
}

}  // namespace

int join_fwd_launch(const JoinArgs& a, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int v = piece_of(a, {a.o, a.a, a.x, a.x_out, a.n_out});
    const bool wide = a.H * a.d > 4096;
    return a.f32 ? dispatch<float>(a, v, wide, st) : dispatch<__nv_bfloat16>(a, v, wide, st);
}

int join_bwd_launch(const JoinBwdArgs& b, void* stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int v = piece_of(b.f, {b.f.o, b.f.a, b.f.x, b.d_x_out, b.d_n, b.d_o, b.d_a, b.d_x});
    const bool wide = b.f.H * b.f.d > 4096;
    return b.f.f32 ? dispatch<float>(b, v, wide, st) : dispatch<__nv_bfloat16>(b, v, wide, st);
}

}  // namespace e2ttt

using namespace e2ttt;

namespace {

int check(const e2ttt_join_params* p) {
    if (!p) return E2TTT_ERR_NULL;
    if (p->io_dtype != E2TTT_F32 && p->io_dtype != E2TTT_BF16) return E2TTT_ERR_DTYPE;
    if (p->B <= 0 || p->H <= 0 || p->L <= 0 || p->d <= 0) return E2TTT_ERR_SHAPE;
    if (p->L > (1 << 30)) return E2TTT_ERR_SHAPE;  // positions are stepped on in 32 bits
    if ((int64_t)p->H * p->d > kJoinMaxWidth || (int64_t)p->B * p->L > (int64_t)1 << 40) return E2TTT_ERR_SHAPE;
    if (p->gate != E2TTT_GATE_NONE && p->gate != E2TTT_GATE_SIGMOID && p->gate != E2TTT_GATE_SILU) return E2TTT_ERR_SHAPE;
    if (!(p->post_eps >= 0.0f) || !(p->pre_eps >= 0.0f)) return E2TTT_ERR_SHAPE;
    return E2TTT_OK;
}

bool io_aligned(const e2ttt_join_params* p, std::initializer_list<const void*> ptrs) {
    for (const void* x : ptrs)
        if (!aligned(x, p->io_dtype == E2TTT_F32 ? 4 : 2)) return false;
    return true;
}
bool f32_aligned(std::initializer_list<const void*> ptrs) {
    for (const void* x : ptrs)
        if (!aligned(x, 4)) return false;
    return true;
}

JoinArgs args_of(const e2ttt_join_params* p, const void* o, const void* a, const void* x, const float* w_post, const float* res_scale,
                 const float* w_pre, void* x_out, void* n_out) {
    return {p->B, p->H, p->L, p->d, p->io_dtype == E2TTT_F32, p->gate, p->post_eps, p->pre_eps, o, a, x, w_post, res_scale, w_pre, x_out, n_out};
}

size_t bytes_of(const e2ttt_join_params* p) {
    return kStatusBytes + (size_t)join_bwd_grid((int64_t)p->B * p->L, p->H * p->d) * 2 * p->H * p->d * 4;
}

}  // namespace

extern "C" {

int e2ttt_join_workspace_bytes(const e2ttt_join_params* p, size_t* bytes) {
    if (!bytes) return E2TTT_ERR_NULL;
    const int rc = check(p);
    if (rc) return rc;
    *bytes = bytes_of(p);
    return E2TTT_OK;
}

int e2ttt_join_fwd(const e2ttt_join_params* p, const void* o, const void* a, const void* x, const float* w_post, const float* res_scale,
                   const float* w_pre, void* x_out, void* n_out, void* stream) {
    int rc = check(p);
    if (rc) return rc;
    if (!o || !x || !w_post || !res_scale || !x_out || !a != (p->gate == E2TTT_GATE_NONE) || !w_pre != !n_out) return E2TTT_ERR_NULL;
    if (!io_aligned(p, {o, a, x, x_out, n_out}) || !f32_aligned({w_post, res_scale, w_pre})) return E2TTT_ERR_ALIGN;
    rc = check_device();
    if (rc) return rc;
    return join_fwd_launch(args_of(p, o, a, x, w_post, res_scale, w_pre, x_out, n_out), stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

int e2ttt_join_bwd(const e2ttt_join_params* p, const void* o, const void* a, const void* x, const float* w_post, const float* res_scale,
                   const float* w_pre, const void* d_x_out, const void* d_n, void* d_o, void* d_a, void* d_x, float* d_w_post,
                   float* d_res_scale, float* d_w_pre, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check(p);
    if (rc) return rc;
    if (!o || !x || !w_post || !res_scale || !d_x_out || !d_o || !d_x || !d_w_post || !d_res_scale) return E2TTT_ERR_NULL;
    const bool gated = p->gate != E2TTT_GATE_NONE;
    if (!a == gated || !d_a == gated || !w_pre != !d_n || !w_pre != !d_w_pre) return E2TTT_ERR_NULL;
    if (!io_aligned(p, {o, a, x, d_x_out, d_n, d_o, d_a, d_x}) || !f32_aligned({w_post, res_scale, w_pre, d_w_post, d_res_scale, d_w_pre}))
        return E2TTT_ERR_ALIGN;
    if (!workspace || workspace_bytes < bytes_of(p)) return E2TTT_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return E2TTT_ERR_ALIGN;
    rc = check_device();
    if (rc) return rc;
    JoinBwdArgs b{args_of(p, o, a, x, w_post, res_scale, w_pre, nullptr, nullptr), d_x_out, d_n, d_o, d_a, d_x, d_w_post, d_res_scale, d_w_pre,
                  reinterpret_cast<float*>(static_cast<char*>(workspace) + kStatusBytes)};
    return join_bwd_launch(b, stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

}  // extern "C"
