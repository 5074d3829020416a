// csrc/dense.hip on the CPU: the host side of the dense operators with a context and kernels that only count what reaches them.
#include <cstdarg>
#include <cstdio>
#include <vector>

#include "dense.hip"

struct legend_ctx {
    CtxView view;
    bool fatal = false, swap_pending = false;
    std::vector<legend_adamw*> optimisers;
};

static char last_error[512];
static int launches;
static AdamTensor last_tensors[64];
static const void* last_grads[64];

namespace legend {

int fail(int code, const char* fmt, ...) noexcept {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(last_error, sizeof last_error, fmt, ap);
    va_end(ap);
    return code;
}
int ctx_enter(legend_ctx* c, CtxView* v) {
    if (!c) return fail(LEGEND_E_INVAL, "null context");
    if (c->fatal) return fail(LEGEND_E_HIP, "unusable");
    (void)hipSetDevice(c->view.device);
    *v = c->view;
    return LEGEND_OK;
}
int ctx_tables_current(legend_ctx* c, bool recording) {
    if (recording && c->swap_pending) return fail(LEGEND_E_STATE, "swap");
    c->swap_pending = false;
    return LEGEND_OK;
}
void ctx_failed(legend_ctx* c) { c->fatal = true; }
void ctx_keep(legend_ctx* c, legend_adamw* o, bool attach) {
    if (attach) c->optimisers.push_back(o);
    else c->optimisers.erase(std::remove(c->optimisers.begin(), c->optimisers.end(), o), c->optimisers.end());
}
int norm_parts(int64_t rows, int32_t) { return (int)(rows < 512 ? rows : 512); }
hipError_t launch_norm_forward(hipStream_t, const NormParams&) { ++launches; return hipSuccess; }
hipError_t launch_norm_backward(hipStream_t, const NormParams&) { ++launches; return hipSuccess; }
int adam_unit_elems(int64_t) { return 1024; }
void adam_state_at(AdamState* s, int64_t steps, double, double) { *s = AdamState{}; s->steps = steps; }
hipError_t launch_adamw(hipStream_t, const AdamParams& a) {
    // every unit belongs to its tensor and every tensor is covered
    int64_t u = 0;
    for (int k = 0; u < a.units && k < 64; ++k) {
        last_tensors[k] = a.tensors[k];
        last_grads[k] = a.grads[k];
        if (a.tensors[k].first_unit != u) return hipErrorInvalidValue;
        for (int64_t left = a.tensors[k].count; left > 0; left -= a.unit_elems)
            if (a.unit_tensor[u++] != k) return hipErrorInvalidValue;
    }
    ++launches;
    a.state->steps += 1;
    return hipSuccess;
}

}  // namespace legend

extern "C" {
const char* legend_last_error(void) { return last_error; }
legend_ctx* stub_context(int dim, int64_t nodes, int relations) {
    legend_ctx* c = new legend_ctx;
    c->view.device = 1;
    c->view.dim = dim;
    c->view.num_nodes = c->view.rows_per_partition = nodes;
    c->view.relation_rows = relations;
    return c;
}
void stub_context_gone(legend_ctx* c) {
    for (legend_adamw* o : c->optimisers) adamw_orphan(o);
    delete c;
}
void stub_set(legend_ctx* c, int recording, int no_memory, int swap_pending) {
    stub_recording = recording != 0;
    stub_no_memory = no_memory != 0;
    c->swap_pending = swap_pending != 0;
}
int stub_launches(void) { return launches; }
int stub_live(void) { return stub_allocations; }
int stub_current_device(void) { return stub_device; }
const void* stub_grad(int k) { return last_grads[k]; }
}
