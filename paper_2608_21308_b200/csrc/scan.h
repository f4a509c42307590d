// Gated linear recurrence: arguments of the launchers, layout of the workspace.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace e2ttt {

constexpr int kScanCh = 64;    // channels of a CTA: a lane has two neighbouring ones
constexpr int kScanSpan = 64;  // tokens between two saved states

struct ScanShape {
    int B, L, D;
    int f32, gate, unit;
    constexpr int64_t blocks() const { return (D + kScanCh - 1) / kScanCh; }
    constexpr int64_t spans() const { return ((int64_t)L + kScanSpan - 1) / kScanSpan; }
};

// CTAs that share a block of channels of a sequence, the CTAs of a cluster: the number with the shortest way through, in turns of a tile per CTA.  kFit clusters of 1 to 8 CTAs
// are on the GPU at a time with two CTAs on an SM (as the driver counts them; half of that with one).  Measured, in the forward with bf16 I/O: a turn takes 3.7 to 4.1 us
// where an SM has two CTAs, 2.1 (one CTA) to 2.8 us (a cluster of eight) where it has one, and a round of clusters some 0.8 turns more to start and to end.  The reverse pass and
// fp32 I/O go by the same figures, and the choice is the best of 1 to 8 or, with fp32 I/O, up to 12 % behind it.
inline int scan_parts(const ScanShape& s, int tile, int on_sm) {
    constexpr int kFit[8] = {296, 148, 93, 71, 56, 45, 37, 33};
    constexpr float kAlone[8] = {0.53f, 0.64f, 0.65f, 0.66f, 0.67f, 0.68f, 0.69f, 0.69f}, kPair[8] = {0.95f, 1.0f, 1.0f, 1.0f, 1.01f, 1.02f, 1.03f, 1.03f};
    const int64_t units = s.B * s.blocks(), tiles = ((int64_t)s.L + tile - 1) / tile;
    int best = 1;
    float least = 0.0f;
    for (int i = 0; i < 8 && i < tiles; ++i) {
        const int64_t fit = kFit[i] * on_sm / 2, whole = units / fit, rest = units - whole * fit;
        const float turns = (float)((tiles + i) / (i + 1)) + 0.8f, one = on_sm == 1 ? kAlone[i] : kPair[i];
        const float way = turns * ((float)whole * one + (rest == 0 ? 0.0f : 2 * rest <= fit ? kAlone[i] : one));
        if (i == 0 || way < least) {
            least = way;
            best = i + 1;
        }
    }
    return best;
}

// CTAs of the reverse pass that share a block of channels, along the tokens
int scan_bwd_parts(const ScanShape& s);

struct ScanLayout {  // byte offsets
    size_t states;   // [B][spans][D] fp32: the state before every 64th token
    size_t rates;    // [B parts][D] fp32: partial sums of d_rate
    size_t codes;    // [tensors][B][blocks][64 spans][64] bytes: x, a_decay, a_in of a block of channels, token after token
    size_t scales;   // [tensors][B][blocks][64 spans][2] bytes
    size_t code_step, scale_step;  // from one tensor to the next
    size_t total;
};
ScanLayout scan_layout(const ScanShape& s, int save);

struct ScanArgs {
    ScanShape s;
    const void *x, *r, *g;  // g: null without an input gate
    const float* rate;
    const uint8_t* starts;  // may be null
    const float* h_init;    // may be null
    void* h;                // null: only the states are wanted
    float* h_final;         // null with h
    float* states;          // null: not saved
    uint8_t *codes, *scales;  // null: inputs not kept in 8 bits
    size_t code_step, scale_step;
    long long wait_cycles;  // after which a device-side wait gives up; 0: at once
};

struct ScanBwdArgs {
    ScanArgs f;  // with codes: x, r and g come from there
    const void* d_h;
    const float* dh_final;  // may be null
    void *d_x, *d_r, *d_g;
    float *d_rate, *dh_init, *part;
};

// return a cudaError_t value as int
int scan_fwd_launch(const ScanArgs& a, void* stream);
int scan_bwd_launch(const ScanBwdArgs& a, void* stream);
int scan_step_launch(const ScanArgs& a, void* stream);

}  // namespace e2ttt
