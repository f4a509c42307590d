// Entry points of the gated linear recurrence: argument checks, workspace, launches.
#include <initializer_list>

#include "api_checks.h"
#include "scan.h"
#include "sm100.cuh"

namespace e2ttt {

ScanLayout scan_layout(const ScanShape& s, int save) {
    ScanLayout l{};
    if (save == E2TTT_SAVE_NONE) return l;
    auto round = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t tensors = save == E2TTT_SAVE_PACKED ? (s.gate ? 3 : 2) : 0, rows = (size_t)s.B * s.blocks() * s.spans() * kScanSpan;
    l.states = kStatusBytes;
    l.rates = l.states + round((size_t)s.B * s.spans() * s.D * 4);
    l.codes = l.rates + round((size_t)s.B * scan_bwd_parts(s) * s.D * 4);
    l.code_step = rows * kScanCh;
    l.scales = l.codes + tensors * l.code_step;
    l.scale_step = rows * 2;
    l.total = l.scales + round(tensors * l.scale_step);
    return l;
}

}  // namespace e2ttt

using namespace e2ttt;

namespace {

int check(const e2ttt_scan_params* p, ScanShape* s) {
    if (!p) return E2TTT_ERR_NULL;
    if (p->io_dtype != E2TTT_F32 && p->io_dtype != E2TTT_BF16) return E2TTT_ERR_DTYPE;
    if (p->B <= 0 || p->L <= 0 || p->D <= 0 || p->D > (1 << 20) || p->L > (1 << 30)) return E2TTT_ERR_SHAPE;
    if (p->gate != E2TTT_GATE_NONE && p->gate != E2TTT_GATE_SIGMOID) return E2TTT_ERR_SHAPE;
    if (p->unit_scale != 0 && p->unit_scale != 1) return E2TTT_ERR_SHAPE;
    *s = ScanShape{p->B, p->L, p->D, p->io_dtype == E2TTT_F32, p->gate == E2TTT_GATE_SIGMOID, p->unit_scale};
    if ((int64_t)p->B * s->blocks() > (int64_t)1 << 24) return E2TTT_ERR_SHAPE;
    if ((int64_t)p->B * p->L > ((int64_t)1 << 40) / p->D) return E2TTT_ERR_SHAPE;
    return E2TTT_OK;
}

bool element_aligned(const ScanShape& s, std::initializer_list<const void*> io, std::initializer_list<const void*> f32) {
    for (const void* p : io)
        if (!aligned(p, s.f32 ? 4 : 2)) return false;
    for (const void* p : f32)
        if (!aligned(p, 4)) return false;
    return true;
}

bool known(int save) { return save == E2TTT_SAVE_NONE || save == E2TTT_SAVE_STATES || save == E2TTT_SAVE_PACKED; }

int check_workspace(const void* ws, size_t bytes, size_t need) {
    if (!need) return E2TTT_OK;
    if (!ws || bytes < need) return E2TTT_ERR_WORKSPACE;
    return aligned(ws, 256) ? E2TTT_OK : E2TTT_ERR_ALIGN;
}

thread_local long long wait_cycles = sm100::kWaitCycles;  // of this host thread's calls

void place(ScanArgs* a, const ScanLayout& l, void* workspace, int save) {
    char* ws = static_cast<char*>(workspace);
    if (save != E2TTT_SAVE_NONE) a->states = reinterpret_cast<float*>(ws + l.states);
    if (save != E2TTT_SAVE_PACKED) return;
    a->codes = reinterpret_cast<uint8_t*>(ws + l.codes);
    a->scales = reinterpret_cast<uint8_t*>(ws + l.scales);
    a->code_step = l.code_step;
    a->scale_step = l.scale_step;
}

}  // namespace

extern "C" {

int e2ttt_scan_workspace_bytes(const e2ttt_scan_params* p, int save, size_t* bytes) {
    ScanShape s;
    if (!bytes) return E2TTT_ERR_NULL;
    const int rc = check(p, &s);
    if (rc) return rc;
    if (!known(save)) return E2TTT_ERR_SHAPE;
    *bytes = scan_layout(s, save).total;
    return E2TTT_OK;
}

int e2ttt_scan_fwd(const e2ttt_scan_params* p, const void* x, const void* a_decay, const void* a_in, const float* rate,
                   const uint8_t* starts, const float* h_init, void* h, float* h_final, void* workspace, size_t workspace_bytes,
                   int save, void* stream) {
    ScanArgs a{};
    int rc = check(p, &a.s);
    if (rc) return rc;
    if (!known(save)) return E2TTT_ERR_SHAPE;
    if (!x || !a_decay || !a_in != !a.s.gate || !rate || !h || !h_final) return E2TTT_ERR_NULL;
    if (!element_aligned(a.s, {x, a_decay, a_in, h}, {rate, h_init, h_final})) return E2TTT_ERR_ALIGN;
    const ScanLayout l = scan_layout(a.s, save);
    rc = check_workspace(workspace, workspace_bytes, l.total);
    if (rc) return rc;
    rc = check_device();
    if (rc) return rc;
    a.x = x; a.r = a_decay; a.g = a_in; a.rate = rate; a.starts = starts; a.h_init = h_init; a.h = h; a.h_final = h_final;
    a.wait_cycles = wait_cycles;
    place(&a, l, workspace, save);
    return scan_fwd_launch(a, stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

int e2ttt_scan_bwd(const e2ttt_scan_params* p, const void* x, const void* a_decay, const void* a_in, const float* rate,
                   const uint8_t* starts, const float* h_init, const void* d_h, const float* dh_final, void* d_x, void* da_decay,
                   void* da_in, float* d_rate, float* dh_init, void* workspace, size_t workspace_bytes, int saved, void* stream) {
    ScanBwdArgs b{};
    int rc = check(p, &b.f.s);
    if (rc) return rc;
    const ScanShape& s = b.f.s;
    if (!known(saved)) return E2TTT_ERR_SHAPE;
    if (saved != E2TTT_SAVE_PACKED && (!x || !a_decay || !a_in != !s.gate)) return E2TTT_ERR_NULL;
    if (!rate || !d_h || !d_x || !da_decay || !da_in != !s.gate || !d_rate || !dh_init) return E2TTT_ERR_NULL;
    if (!element_aligned(s, {x, a_decay, a_in, d_h, d_x, da_decay, da_in}, {rate, h_init, dh_final, d_rate, dh_init})) return E2TTT_ERR_ALIGN;
    const int save = saved == E2TTT_SAVE_NONE ? (int)E2TTT_SAVE_STATES : saved;
    const ScanLayout l = scan_layout(s, save);
    rc = check_workspace(workspace, workspace_bytes, l.total);
    if (rc) return rc;
    rc = check_device();
    if (rc) return rc;
    b.f.x = x; b.f.r = a_decay; b.f.g = a_in; b.f.rate = rate; b.f.starts = starts; b.f.h_init = h_init;
    b.f.wait_cycles = wait_cycles;
    place(&b.f, l, workspace, save);
    if (saved == E2TTT_SAVE_NONE && scan_fwd_launch(b.f, stream) != 0) return E2TTT_ERR_CUDA;
    b.d_h = d_h; b.dh_final = dh_final; b.d_x = d_x; b.d_r = da_decay; b.d_g = da_in; b.d_rate = d_rate; b.dh_init = dh_init;
    b.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + l.rates);
    return scan_bwd_launch(b, stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

int e2ttt_scan_step(const e2ttt_scan_params* p, const void* x, const void* a_decay, const void* a_in, const float* rate,
                    const uint8_t* starts, const float* h_state, void* h, float* h_out, void* stream) {
    ScanArgs a{};
    int rc = check(p, &a.s);
    if (rc) return rc;
    if (!x || !a_decay || !a_in != !a.s.gate || !rate || !h_state || !h || !h_out) return E2TTT_ERR_NULL;
    if (!element_aligned(a.s, {x, a_decay, a_in, h}, {rate, h_state, h_out})) return E2TTT_ERR_ALIGN;
    rc = check_device();
    if (rc) return rc;
    a.x = x; a.r = a_decay; a.g = a_in; a.rate = rate; a.starts = starts; a.h_init = h_state; a.h = h; a.h_final = h_out;
    return scan_step_launch(a, stream) == 0 ? E2TTT_OK : E2TTT_ERR_CUDA;
}

int e2ttt_selftest_scan_wait_limit(long long limit_cycles) {
    if (limit_cycles > sm100::kWaitCycles) return E2TTT_ERR_SHAPE;
    wait_cycles = limit_cycles < 0 ? sm100::kWaitCycles : limit_cycles;
    return E2TTT_OK;
}

}  // extern "C"
