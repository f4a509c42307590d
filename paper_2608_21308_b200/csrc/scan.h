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

// CTAs that share a block of channels of a sequence: as many as fill the GPU's 148 SMs once, `on_sm` on each, up to a cluster of eight and a tile each.  All of them run
// at once then: a second, part-filled round of CTAs that walk a whole sequence would take as long as the first.
inline int scan_parts(const ScanShape& s, int tile, int on_sm) {
    const int64_t fit = 148 * on_sm / (s.B * s.blocks()), tiles = ((int64_t)s.L + tile - 1) / tile, parts = fit < tiles ? fit : tiles;
    return (int)(parts < 1 ? 1 : parts > 8 ? 8 : parts);
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
