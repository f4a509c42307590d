// Block join (norm after a block, gate, residual scale and sum, norm before the next block): arguments of the launchers.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace e2ttt {

constexpr int kJoinMaxWidth = 8192;  // H d: 16 values a thread, 512 threads

struct JoinArgs {
    int B, H, L, d;
    int f32, gate;  // gate: e2ttt_gate
    float post_eps, pre_eps;
    const void *o, *a, *x;                        // a may be null (no gate)
    const float *w_post, *res_scale, *w_pre;      // w_pre may be null (no second norm)
    void *x_out, *n_out;                          // n_out: null with w_pre
    uint8_t* packed;                              // o, x and a in 8 bits (JoinPacked); null: not kept, or (reverse pass) not read
};

// Where the packed inputs lie: codes of o, x and, with a gate, a as rows of H d columns filled up to blocks of 32, then their scales, rows filled up to words.
struct JoinPacked {
    int64_t code_row, scale_row;    // bytes of a row
    int64_t code_step, scale_step;  // bytes of a tensor
    int64_t scales, total;          // where the scales start; bytes in all
};
inline JoinPacked join_packed(int64_t tokens, int width, int tensors) {
    JoinPacked l{};
    l.code_row = (width + 31) / 32 * 32;
    l.scale_row = (l.code_row / 32 + 3) / 4 * 4;
    l.code_step = tokens * l.code_row;
    l.scale_step = tokens * l.scale_row;
    l.scales = tensors * l.code_step;
    l.total = l.scales + tensors * l.scale_step;
    return l;
}

struct JoinBwdArgs {
    JoinArgs f;
    const void *d_x_out, *d_n;                    // d_n: null with w_pre
    void *d_o, *d_a, *d_x;
    float *d_w_post, *d_res_scale, *d_w_pre;
    float* part;                                  // [grid][2][H d]
};

// CTAs of the reverse pass, each with partial sums of the parameters' gradients: 512 threads on an SM, a thread per 8 columns (16 above 4096 columns)
inline int join_bwd_grid(int64_t tokens, int width) {
    const int threads = width <= 4096 ? (width + 255) / 256 * 32 : 512;
    const int most = 148 * (threads <= 64 ? 8 : 512 / threads);
    return (int)(tokens < most ? tokens : most);
}

// return a cudaError_t value as int
int join_fwd_launch(const JoinArgs& a, void* stream);
int join_bwd_launch(const JoinBwdArgs& a, void* stream);

}  // namespace e2ttt
