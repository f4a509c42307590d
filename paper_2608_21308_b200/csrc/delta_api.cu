// Entry points of the gated delta rule: argument checks, workspace, launches.
#include <initializer_list>

#include "api_checks.h"
#include "delta.h"

using namespace e2ttt;

namespace {

int check(const e2ttt_delta_params* p, DeltaShape* s) {
    if (!p) return E2TTT_ERR_NULL;
    if (p->io_dtype != E2TTT_F32 && p->io_dtype != E2TTT_BF16) return E2TTT_ERR_DTYPE;
    if (p->B <= 0 || p->H <= 0 || p->Hk <= 0 || p->L <= 0 || p->dk <= 0 || p->dv <= 0) return E2TTT_ERR_SHAPE;
    if (p->H % p->Hk || p->dk > kDeltaMaxD || p->dv > kDeltaMaxD || p->L > (1 << 30)) return E2TTT_ERR_SHAPE;
    if ((int64_t)p->B * p->H > (int64_t)1 << 24) return E2TTT_ERR_SHAPE;
    // the kernels' grids: a warp per chunk, a CTA per block of 64 tokens
    const int64_t nch = ((int64_t)p->L + kDeltaChunk - 1) / kDeltaChunk;
    if ((int64_t)p->B * p->H * nch > (int64_t)1 << 30) return E2TTT_ERR_SHAPE;
    if (!(p->scale - p->scale == 0.0f)) return E2TTT_ERR_SHAPE;  // not finite
    *s = DeltaShape{p->B, p->H, p->Hk, p->L, p->dk, p->dv, p->io_dtype == E2TTT_F32, p->scale};
    return E2TTT_OK;
}

int check_workspace(const void* ws, size_t bytes, size_t need) {
    if (!ws || bytes < need) return E2TTT_ERR_WORKSPACE;
    return aligned(ws, 256) ? E2TTT_OK : E2TTT_ERR_ALIGN;
}

// elements of io_dtype and fp32 at the alignment that their loads need
bool element_aligned(const DeltaShape& s, std::initializer_list<const void*> io, std::initializer_list<const void*> f32) {
    for (const void* p : io)
        if (!aligned(p, s.f32 ? 4 : 2)) return false;
    for (const void* p : f32)
        if (!aligned(p, 4)) return false;
    return true;
}

}  // namespace

extern "C" {

int e2ttt_delta_workspace_bytes(const e2ttt_delta_params* p, int save_states, size_t* bytes) {
    DeltaShape s;
    if (!bytes) return E2TTT_ERR_NULL;
    const int rc = check(p, &s);
    if (rc) return rc;
    *bytes = delta_layout(s, save_states != 0).total;
    return E2TTT_OK;
}

int e2ttt_delta_fwd(const e2ttt_delta_params* p, const void* q, const void* k, const void* v, const float* eta,
                    const float* log_gamma, const float* S_init, void* o, float* S_final, void* workspace, size_t workspace_bytes,
                    int save_states, void* stream) {
    DeltaShape s;
    int rc = check(p, &s);
    if (rc) return rc;
    if (!q || !k || !v || !eta || !log_gamma || !o || !S_final) return E2TTT_ERR_NULL;
    if (!element_aligned(s, {q, k, v, o}, {eta, log_gamma, S_init, S_final})) return E2TTT_ERR_ALIGN;
    DeltaArgs a{s, delta_layout(s, save_states != 0), q, k, v, eta, log_gamma, S_init, o, S_final, static_cast<char*>(workspace),
                save_states != 0};
    rc = check_workspace(workspace, workspace_bytes, a.l.total);
    if (rc) return rc;
    rc = check_device();
    if (rc) return rc;
    if (delta_prep_launch(a, stream) != 0 || delta_fwd_launch(a, stream) != 0) return E2TTT_ERR_CUDA;
    return E2TTT_OK;
}

int e2ttt_delta_bwd(const e2ttt_delta_params* p, const void* q, const void* k, const void* v, const float* eta,
                    const float* log_gamma, const float* S_init, const void* d_o, const float* dS_final, void* dq, void* dk, void* dv,
                    float* d_eta, float* d_log_gamma, float* dS_init, void* workspace, size_t workspace_bytes, int states_saved,
                    void* stream) {
    DeltaShape s;
    int rc = check(p, &s);
    if (rc) return rc;
    if (!q || !k || !v || !eta || !log_gamma || !d_o || !dq || !dk || !dv || !d_eta || !d_log_gamma || !dS_init) return E2TTT_ERR_NULL;
    if (!element_aligned(s, {q, k, v, d_o, dq, dk, dv}, {eta, log_gamma, S_init, dS_final, d_eta, d_log_gamma, dS_init}))
        return E2TTT_ERR_ALIGN;
    DeltaBwdArgs b{DeltaArgs{s, delta_layout(s, true), q, k, v, eta, log_gamma, S_init, nullptr, nullptr, static_cast<char*>(workspace), 1},
                   d_o, dS_final, dq, dk, dv, d_eta, d_log_gamma, dS_init};
    rc = check_workspace(workspace, workspace_bytes, b.f.l.total);
    if (rc) return rc;
    rc = check_device();
    if (rc) return rc;
    if (!states_saved && (delta_prep_launch(b.f, stream) != 0 || delta_fwd_launch(b.f, stream) != 0)) return E2TTT_ERR_CUDA;
    return delta_bwd_launch(b, stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

int e2ttt_delta_step(const e2ttt_delta_params* p, const void* q, const void* k, const void* v, const float* eta,
                     const float* log_gamma, const float* S, void* o, float* S_out, void* stream) {
    DeltaStepArgs a{};
    int rc = check(p, &a.s);
    if (rc) return rc;
    if (!q || !k || !v || !eta || !log_gamma || !S || !o || !S_out) return E2TTT_ERR_NULL;
    if (!element_aligned(a.s, {q, k, v, o}, {eta, log_gamma, S, S_out})) return E2TTT_ERR_ALIGN;
    a.q = q; a.k = k; a.v = v; a.eta = eta; a.log_gamma = log_gamma; a.S = S; a.o = o; a.S_out = S_out;
    rc = check_device();
    if (rc) return rc;
    return delta_step_launch(a, stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

}  // extern "C"
