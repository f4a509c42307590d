// Gated delta rule: arguments of the launchers and the layout of the workspace (no CUDA types: the host tests read it too).
//
// Per sequence and value head a state S [dv, dk] moves token by token:
//   S'_t = g_t S_{t-1},  e_t = v_t - S'_t k_t,  S_t = S'_t + eta_t e_t k_t^T,  o_t = scale S_t q_t,   g_t = exp(log_gamma_t).
// A chunk of 32 tokens from its start state S_0 in matrix form, b_t the product of g up to token t, D_ti = b_t / b_i:
//   P = V - b S_0 K,   e = T P,  T = (I + strict(D (K K^T)) eta)^-1,   u = eta e,
//   O = b scale S_0 Q + A u,  A = scale lower(D (Q K^T)),   S = b_end S_0 + (D_end u)^T K.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace e2ttt {

constexpr int kDeltaChunk = 32;  // tokens per chunk: a warp's row for its gates, two k-steps of the MMAs
constexpr int kDeltaBlock = 64;  // tokens per saved state: two chunks
constexpr int kDeltaMaxD = 128;  // a slice of 16 state rows of 128 columns is a quarter of a warp's registers
// A chunk's record: T and A eta (two fp16 terms each, 2 KB a term), eight rows of 32 floats; with saved states also A and the T of the reverse
// pass, (I + eta strict(D (K K^T)))^-1, and A and strict(D (K K^T)) in fp32, in the order of a product's six 16 x 8 tiles on and below the diagonal blocks.
// The forward fetches the first 9 KB, the reverse walk 9 KB from the scalars on; the fp32 matrices are for the decays' gradients.
constexpr int kDeltaRecBytes = 9216;
constexpr int kDeltaRecSkip = 8192;
constexpr int kDeltaRecPairs = 17408;
// rows of a record's scalars: b of K and Q (with the scales of their tiles), eta, D_end, eta D_end, eta b
enum { kRecBk = 0, kRecBq = 1, kRecEta = 2, kRecDend = 3, kRecW = 4, kRecZ = 5, kRecHead = 7 };
// the last row: decay of the whole chunk; what undoes the scales of T, A eta, K, Q, the reverse pass' T and A; then bounds of the chunk's
// operands: max b |k| (2-norm), row sums of T, max |eta| D_end (in units of the K tile), sum |eta| D_end |k|
enum { kHeadEnd = 0, kHeadT = 1, kHeadA = 2, kHeadK = 3, kHeadQ = 4, kHeadR = 5, kHeadKn = 6, kHeadTsum = 7, kHeadAr = 8, kHeadWmax = 9, kHeadWsum = 10,
       // and of the reverse pass: max D_end |k|, column sums of its T, max |eta| b (in units of the K tile), sum |eta| b |k|, sum b scale |q|
       kHeadKe = 11, kHeadRsum = 12, kHeadZmax = 13, kHeadZsum = 14, kHeadQsum = 15 };

struct DeltaShape {
    int B, H, Hk, L, dk, dv;
    int f32;  // 1: fp32 I/O
    float scale;
};

struct DeltaLayout {
    int DK;            // columns of a padded state row: 64 or 128
    int terms;         // fp16 terms of a query or key: 1 (bf16 I/O, exact) or 2
    int dvp;           // value rows padded to 16
    int slices;        // dvp / 16: warps that a sequence's state is cut into
    int nch, nblk;     // chunks of 32 tokens, blocks of 64
    int64_t N, Nk;     // sequences (value heads), query / key heads
    size_t qk_bytes;   // query and key tiles of a chunk
    size_t rec_bytes;  // record of a chunk
    size_t state_bytes;  // a slice of a state: one term of its fragments
    // offsets in bytes.  Saved for the reverse pass, all in fragment order (a lane's 16 bytes of one product's A operand together), per slice:
    // the state before every block (first terms and second terms), e of every chunk, S Q^T and S K^T of the state before it in
    // fp32 (at the state's scale); by its chain: X behind every block, dP of every chunk; what undoes the scales; per token, sums over a slice's rows
    size_t qk, rec, S, S_lo, s_inv, e, e_inv, sq, sk, c_inv, X, x_inv, dp, dp_lo, dp_inv, max_do, part_eta, part_s, part_x, hx, total;
};

inline DeltaLayout delta_layout(const DeltaShape& s, bool save) {
    DeltaLayout l{};
    l.DK = s.dk <= 64 ? 64 : 128;
    l.terms = s.f32 ? 2 : 1;
    l.dvp = (s.dv + 15) / 16 * 16;
    l.slices = l.dvp / 16;
    l.nch = (int)(((int64_t)s.L + kDeltaChunk - 1) / kDeltaChunk);
    l.nblk = (int)(((int64_t)s.L + kDeltaBlock - 1) / kDeltaBlock);
    l.N = (int64_t)s.B * s.H;
    l.Nk = (int64_t)s.B * s.Hk;
    l.qk_bytes = (size_t)2 * l.terms * 64 * l.DK;
    l.rec_bytes = save ? kDeltaRecPairs + 2 * 3072 : kDeltaRecBytes;
    l.state_bytes = (size_t)32 * l.DK;
    size_t at = 256;  // the status block
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    l.qk = take((size_t)l.Nk * l.nch * l.qk_bytes);
    l.rec = take((size_t)l.N * l.nch * l.rec_bytes);
    if (save) {
        const size_t chunks = (size_t)l.N * l.nch * l.slices, blocks = (size_t)l.N * l.nblk * l.slices;
        l.S = take(blocks * l.state_bytes);
        l.S_lo = take(blocks * l.state_bytes);
        l.s_inv = take(blocks * 4);
        l.e = take(chunks * 2048);
        l.e_inv = take(chunks * 4);
        l.sq = take(chunks * 2048);
        l.sk = take(chunks * 2048);
        l.c_inv = take(chunks * 4);
        l.X = take(blocks * l.state_bytes * l.terms);
        l.x_inv = take(blocks * 4);
        l.dp = take(chunks * 1024 * l.terms);
        l.dp_lo = l.terms == 1 ? take(chunks * 1024) : 0;  // apart: dq and dk are of first terms with bf16
        l.dp_inv = take(chunks * 4);
        l.max_do = take(chunks * 4);
        l.part_eta = take(chunks * kDeltaChunk * 4);
        l.part_s = take(chunks * kDeltaChunk * 4);
        l.part_x = take(chunks * kDeltaChunk * 4);
        l.hx = take((size_t)l.N * l.nblk * l.slices * 16);
    }
    l.total = at;
    return l;
}

// Slices of a sequence that share a CTA and the tiles that it fetches: as many as leave 96 CTAs, shared out evenly (five are 3 and 2, not 4 and 1).
// 300 sequences of 512 tokens, bf16, us a call, evenly and not: values of 16: 130 and 151 with keys of 128, 77 and 107 with 64; values of 80: 214 and 218.
inline int slices_per_cta(const DeltaLayout& l, int most) {
    int per = most;
    while (per > 1 && l.N * ((l.slices + per - 1) / per) < 96) per >>= 1;
    const int ctas = (l.slices + per - 1) / per;
    return (l.slices + ctas - 1) / ctas;
}

struct DeltaArgs {
    DeltaShape s;
    DeltaLayout l;
    const void *q, *k, *v;
    const float *eta, *log_gamma, *S_init;  // S_init may be null
    void* o;                                // may be null (recomputation)
    float* S_final;                         // may be null (recomputation)
    char* ws;
    int save;
};

struct DeltaBwdArgs {
    DeltaArgs f;
    const void* d_o;
    const float* dS_final;  // may be null
    void *dq, *dk, *dv;
    float *d_eta, *d_log_gamma, *dS_init;
};

struct DeltaStepArgs {
    DeltaShape s;
    const void *q, *k, *v;
    const float *eta, *log_gamma, *S;
    void* o;
    float* S_out;
};

// return a cudaError_t value as int
int delta_prep_launch(const DeltaArgs& a, void* stream);
int delta_fwd_launch(const DeltaArgs& a, void* stream);
int delta_bwd_launch(const DeltaBwdArgs& a, void* stream);
int delta_step_launch(const DeltaStepArgs& a, void* stream);

}  // namespace e2ttt
