// Host side of the operators on the caller's own tensors (layer norm, AdamW): argument checks, the optimiser's tables,
// enqueueing on the context's compute stream.  Nothing here allocates device memory or waits on the way of a forward, backward or step call,
// but for the first call on table rows after a swap, which sends the partition table (ctx_tables_current).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

#include "host_guard.h"
#include "legend_internal.h"

using namespace legend;

struct legend_adamw {
    legend_ctx* ctx = nullptr;              // null once the context is destroyed
    int device = 0;
    legend_adamw_config cfg{};
    std::vector<legend_adamw_tensor> tensors;
    char* mem = nullptr;                    // everything below, one allocation
    AdamTensor* d_tensors = nullptr;
    const void** d_grads = nullptr;
    int32_t* d_unit_tensor = nullptr;
    AdamState* d_state = nullptr;
    double* d_partial = nullptr;
    int64_t units = 0;
    int32_t unit_elems = 0;
    bool stream = false;
    int32_t kinds = 0;
    std::vector<std::pair<uintptr_t, uintptr_t>> used;      // memory of tensors, states and gradients: disjoint, in order
};

namespace {

#define DENSE_TRY(c, expr)                                                                                    \
    do {                                                                                                      \
        hipError_t _e = (expr);                                                                               \
        if (_e != hipSuccess) {                                                                               \
            ctx_failed(c);                                                                                    \
            return fail(LEGEND_E_HIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(_e), __FILE__, __LINE__); \
        }                                                                                                     \
    } while (0)

// The calling thread's current device comes back when the call ends.
struct DeviceScope {
    int before = -1;
    DeviceScope() { if (hipGetDevice(&before) != hipSuccess) before = -1; }
    ~DeviceScope() {
        int now = -1;
        if (before >= 0 && hipGetDevice(&now) == hipSuccess && now != before) (void)hipSetDevice(before);
    }
};

int recording(legend_ctx* c, hipStream_t st, bool* yes) {
    hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
    DENSE_TRY(c, hipStreamIsCapturing(st, &s));
    *yes = s != hipStreamCaptureStatusNone;
    return LEGEND_OK;
}

struct Range {
    uintptr_t lo, hi;
};
bool meets(const Range& a, const Range& b) { return a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi; }
Range bytes_at(const void* p, int64_t bytes) { return {(uintptr_t)p, p ? (uintptr_t)p + (uintptr_t)bytes : (uintptr_t)p}; }
bool aligned_to(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) == 0; }

// ---- layer norm ---------------------------------------------------------------------------------------------------

struct Matrix {
    const void* p;
    int64_t stride;
    int size;                               // bytes of an element
    Range range;
};

// a matrix argument: its range, the columns between its rows included, or an error
int check_matrix(const char* name, const void* p, int64_t stride, int type, int64_t rows, int dim, bool repeats, Matrix* m) {
    if (!p) return fail(LEGEND_E_INVAL, "%s must not be NULL", name);
    const int size = type_size(type);
    if (!aligned_to(p, size)) return fail(LEGEND_E_INVAL, "%s is not aligned to its elements", name);
    if (stride < dim && !(repeats && stride == 0)) return fail(LEGEND_E_INVAL, "%s_stride must be at least dim%s", name, repeats ? " (or 0)" : "");
    if (stride > ((int64_t)1 << 56) / size / std::max<int64_t>(rows, 1)) return fail(LEGEND_E_INVAL, "%s_stride is too large", name);
    *m = {p, stride, size, bytes_at(p, ((rows - 1) * stride + dim) * size)};
    return LEGEND_OK;
}

int norm_params(const CtxView& v, const legend_layer_norm* n, NormParams* out) {
    if (!n) return fail(LEGEND_E_INVAL, "NULL argument");
    if (n->struct_size != sizeof(legend_layer_norm)) return fail(LEGEND_E_INVAL, "legend_layer_norm.struct_size mismatch");
    if (n->dim < 1 || n->dim > kNormMaxDim) return fail(LEGEND_E_INVAL, "dim must be in [1, %d]", kNormMaxDim);
    if (n->rows < 0 || n->rows > ((int64_t)1 << 40)) return fail(LEGEND_E_INVAL, "rows must be in [0, 2^40]");
    if (!type_known(n->x_type)) return fail(LEGEND_E_INVAL, "unknown x_type %d", n->x_type);
    if ((n->weight || n->bias) && !type_known(n->weight_type)) return fail(LEGEND_E_INVAL, "unknown weight_type %d", n->weight_type);
    if (!(n->eps > 0.f) || !std::isfinite(n->eps)) return fail(LEGEND_E_INVAL, "eps must be positive and finite");
    NormParams a{};
    a.rows = n->rows;
    a.dim = n->dim;
    a.eps = n->eps;
    a.x_type = n->x_type;
    if (n->table < 0) {
        a.x = n->x;
        a.x_stride = n->x_stride;
    } else {
        if (n->table != LEGEND_TABLE_NODE_EMB && n->table != LEGEND_TABLE_REL_EMB)
            return fail(LEGEND_E_INVAL, "table must be LEGEND_TABLE_NODE_EMB, LEGEND_TABLE_REL_EMB or -1");
        if (n->x) return fail(LEGEND_E_INVAL, "x must be NULL with a table");
        if (n->x_type != LEGEND_TYPE_FLOAT) return fail(LEGEND_E_INVAL, "x_type must be LEGEND_TYPE_FLOAT with a table");
        if (n->dim != v.dim) return fail(LEGEND_E_INVAL, "dim is %d, the tables have %d", n->dim, v.dim);
        if (!n->status || !aligned_to(n->status, 4)) return fail(LEGEND_E_INVAL, "status must be a word on the device");
        if (!aligned_to(n->ids, 8)) return fail(LEGEND_E_INVAL, "ids are not aligned to their elements");
        a.ids = n->ids;
        a.status = n->status;
        a.rows_per_partition = v.rows_per_partition;
        a.part_base = v.part_emb;
        a.rel_base = n->table == LEGEND_TABLE_REL_EMB ? v.E_rel : nullptr;
        a.table_rows = n->table == LEGEND_TABLE_REL_EMB ? v.relation_rows : v.num_nodes;
    }
    const int ws = type_size(n->weight_type);
    if (!aligned_to(n->weight, ws) || !aligned_to(n->bias, ws)) return fail(LEGEND_E_INVAL, "weight or bias is not aligned to its elements");
    if (!aligned_to(n->mean, 4) || !aligned_to(n->rstd, 4)) return fail(LEGEND_E_INVAL, "mean or rstd is not aligned to its elements");
    a.weight = n->weight;
    a.bias = n->bias;
    a.weight_type = n->weight_type;
    a.mean = n->mean;
    a.rstd = n->rstd;
    *out = a;
    return LEGEND_OK;
}

bool types_go_together(int x_type, int y_type) {
    return type_known(y_type) && (x_type == LEGEND_TYPE_FLOAT || y_type == LEGEND_TYPE_FLOAT || y_type == x_type);
}

// what both directions read besides the matrices
void read_ranges(const legend_layer_norm* n, std::vector<Range>* r) {
    const int64_t wb = (int64_t)n->dim * type_size(n->weight_type);
    r->push_back(bytes_at(n->weight, wb));
    r->push_back(bytes_at(n->bias, wb));
    if (n->table >= 0) r->push_back(bytes_at(n->ids, n->rows * 8));
}

// `written` against one another and against `read`
bool clash(const std::vector<Range>& written, const std::vector<Range>& read) {
    for (size_t i = 0; i < written.size(); ++i) {
        for (size_t j = i + 1; j < written.size(); ++j)
            if (meets(written[i], written[j])) return true;
        for (const Range& r : read)
            if (meets(written[i], r)) return true;
    }
    return false;
}
bool same_place(const Matrix& a, const Matrix& b) { return a.p == b.p && a.size == b.size && a.stride == b.stride; }

// ---- AdamW --------------------------------------------------------------------------------------------------------

int enter_opt(legend_adamw* o, CtxView* v) {
    if (!o) return fail(LEGEND_E_INVAL, "null optimiser");
    if (!o->ctx) return fail(LEGEND_E_STATE, "the optimiser's context has been destroyed");
    return ctx_enter(o->ctx, v);
}

// Memory that a step writes overlaps nothing else that it uses; read-only gradients may share memory.
// `used` receives all of it.
int check_apart(const std::vector<legend_adamw_tensor>& ts, const void* const* grads, std::vector<std::pair<uintptr_t, uintptr_t>>* used) {
    struct Piece {
        uintptr_t lo, hi;
        bool written;
        int64_t tensor;
    };
    std::vector<Piece> all;
    auto add = [&](const void* p, int64_t bytes, bool written, int64_t k) {
        if (p && bytes > 0) all.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written, k});
    };
    for (size_t k = 0; k < ts.size(); ++k) {
        const legend_adamw_tensor& t = ts[k];
        const int64_t state = t.count * (t.state_type == LEGEND_STATE_BLOCK ? 1 : 4);
        const int64_t scales = (t.count + kAdamBlock - 1) / kAdamBlock * 4;
        add(t.param, t.count * type_size(t.param_type), true, (int64_t)k);
        add(t.master, t.count * 4, true, (int64_t)k);
        add(t.m, state, true, (int64_t)k);
        add(t.v, state, true, (int64_t)k);
        add(t.m_scale, scales, true, (int64_t)k);
        add(t.v_scale, scales, true, (int64_t)k);
        add(grads[k], t.count * type_size(t.grad_type), false, (int64_t)k);
    }
    std::sort(all.begin(), all.end(), [](const Piece& a, const Piece& b) { return a.lo < b.lo; });
    // furthest ends so far, of what is written and of everything
    uintptr_t end_written = 0, end_any = 0;
    for (const Piece& p : all) {
        if (p.lo < end_written || (p.written && p.lo < end_any))
            return fail(LEGEND_E_INVAL, "memory of tensor %lld overlaps another tensor, state or gradient", (long long)p.tensor);
        if (p.written) end_written = std::max(end_written, p.hi);
        end_any = std::max(end_any, p.hi);
    }
    used->clear();
    for (const Piece& p : all) {
        if (!used->empty() && p.lo <= used->back().second) used->back().second = std::max(used->back().second, p.hi);
        else used->push_back({p.lo, p.hi});
    }
    return LEGEND_OK;
}

// whether one fp32 at p lies in the optimiser's memory
bool lies_in(const std::vector<std::pair<uintptr_t, uintptr_t>>& used, const float* p) {
    if (!p) return false;
    auto it = std::upper_bound(used.begin(), used.end(), (uintptr_t)p + 3, [](uintptr_t x, const std::pair<uintptr_t, uintptr_t>& r) { return x < r.first; });
    return it != used.begin() && (uintptr_t)p < (--it)->second;
}

int check_tensor(const legend_adamw_tensor& t, int64_t k) {
#define REFUSE(cond, what) if (cond) return fail(LEGEND_E_INVAL, "tensor %lld: %s", (long long)k, what)
    REFUSE(t.count < 0 || t.count > ((int64_t)1 << 48), "count out of range");
    REFUSE(!type_known(t.param_type) || !type_known(t.grad_type), "unknown element type");
    REFUSE(t.state_type != LEGEND_STATE_FLOAT && t.state_type != LEGEND_STATE_BLOCK, "unknown state type");
    REFUSE(t.reserved != 0, "reserved must be 0");
    REFUSE(!(t.weight_decay >= 0.0) || !std::isfinite(t.weight_decay), "weight_decay must be finite and not negative");
    REFUSE(!(t.lr_scale >= 0.0) || !std::isfinite(t.lr_scale), "lr_scale must be finite and not negative");
    REFUSE(t.master && t.param_type == LEGEND_TYPE_FLOAT, "a master copy belongs beside a 16-bit parameter");
    if (t.count == 0) return LEGEND_OK;
    const bool block = t.state_type == LEGEND_STATE_BLOCK;
    REFUSE(!t.param || !t.grad || !t.m || !t.v, "param, grad, m and v must not be NULL");
    REFUSE(block && (!t.m_scale || !t.v_scale), "block states need m_scale and v_scale");
    REFUSE(!block && (t.m_scale || t.v_scale), "m_scale and v_scale belong to block states");
    REFUSE(!aligned_to(t.param, type_size(t.param_type)) || !aligned_to(t.grad, type_size(t.grad_type)) || !aligned_to(t.master, 4) ||
           !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4) || (!block && (!aligned_to(t.m, 4) || !aligned_to(t.v, 4))),
           "a pointer is not aligned to its elements");
#undef REFUSE
    return LEGEND_OK;
}

// Where parameters, states and gradients of all tensors take more than half of the Infinity Cache, a step marks the first two as
// streaming, so that the gradients, which the norm has just read, are still there for it.  (fp32, marked against not: 100 MB 37 and 33 us, where
// everything stays in the cache from step to step; 160 MB 52 and 56, 240 MB 72 and 81, 1.2 GB 312 and 374.)
constexpr int64_t kStreamBytes = (int64_t)128 << 20;
int64_t tensor_bytes(const legend_adamw_tensor& t) {
    return t.count * (type_size(t.param_type) + type_size(t.grad_type) + (t.master ? 4 : 0) + (t.state_type == LEGEND_STATE_BLOCK ? 2 : 8));
}

int refuse_recording(legend_ctx* c, hipStream_t st, const char* what) {
    bool rec = false;
    int rc = recording(c, st, &rec);
    if (rc) return rc;
    return rec ? fail(LEGEND_E_STATE, "%s while the compute stream is recording a graph", what) : LEGEND_OK;
}

}  // namespace

namespace legend {

void adamw_orphan(legend_adamw* opt) { opt->ctx = nullptr; }

}  // namespace legend

extern "C" {

int64_t legend_layer_norm_workspace(int64_t rows, int32_t dim) {
    if (dim < 1 || dim > kNormMaxDim || rows < 0 || rows > ((int64_t)1 << 40)) return -1;
    return (int64_t)norm_parts(rows, dim) * 2 * dim * (int64_t)sizeof(float);
}

int legend_layer_norm_forward(legend_ctx* c, const legend_layer_norm* n) {
    return guarded("legend_layer_norm_forward", [&]() -> int {
    DeviceScope scope;
    CtxView v;
    int rc = ctx_enter(c, &v);
    if (rc) return rc;
    NormParams a;
    rc = norm_params(v, n, &a);
    if (rc) return rc;
    if (!types_go_together(n->x_type, n->y_type)) return fail(LEGEND_E_INVAL, "y_type %d does not go with x_type %d", n->y_type, n->x_type);
    if (n->rows == 0) return LEGEND_OK;
    Matrix x{}, y{};
    if (n->table < 0) {
        rc = check_matrix("x", n->x, n->x_stride, n->x_type, n->rows, n->dim, true, &x);
        if (rc) return rc;
    }
    rc = check_matrix("y", n->y, n->y_stride, n->y_type, n->rows, n->dim, false, &y);
    if (rc) return rc;
    std::vector<Range> written = {y.range, bytes_at(n->mean, n->rows * 4), bytes_at(n->rstd, n->rows * 4)}, read;
    if (n->table >= 0) written.push_back(bytes_at(n->status, 4));
    read_ranges(n, &read);
    bool bad = clash(written, read);
    if (n->table < 0) {
        bad = bad || (meets(y.range, x.range) && !same_place(x, y));
        written.erase(written.begin());
        bad = bad || clash(written, {x.range});
    }
    if (bad) return fail(LEGEND_E_INVAL, "an output overlaps other memory of the call");
    a.y = n->y;
    a.y_stride = n->y_stride;
    a.y_type = n->y_type;
    if (n->table >= 0) {
        bool rec = false;
        rc = recording(c, v.stream, &rec);
        if (rc) return rc;
        rc = ctx_tables_current(c, rec);
        if (rc) return rc;
    }
    DENSE_TRY(c, launch_norm_forward(v.stream, a));
    return LEGEND_OK;
    });
}

int legend_layer_norm_backward(legend_ctx* c, const legend_layer_norm* n) {
    return guarded("legend_layer_norm_backward", [&]() -> int {
    DeviceScope scope;
    CtxView v;
    int rc = ctx_enter(c, &v);
    if (rc) return rc;
    NormParams a;
    rc = norm_params(v, n, &a);
    if (rc) return rc;
    if (!types_go_together(n->x_type, n->dy_type)) return fail(LEGEND_E_INVAL, "dy_type %d does not go with x_type %d", n->dy_type, n->x_type);
    const bool sums = n->dweight || n->dbias;
    if (!sums && !n->dx) return fail(LEGEND_E_INVAL, "none of dx, dweight and dbias is asked for");
    std::vector<Range> written, read;
    if (sums) {
        if (!type_known(n->dweight_type)) return fail(LEGEND_E_INVAL, "unknown dweight_type %d", n->dweight_type);
        if (n->accumulate != 0 && n->accumulate != 1) return fail(LEGEND_E_INVAL, "accumulate must be 0 or 1");
        const int ds = type_size(n->dweight_type);
        if (!aligned_to(n->dweight, ds) || !aligned_to(n->dbias, ds)) return fail(LEGEND_E_INVAL, "dweight or dbias is not aligned to its elements");
        const int64_t need = legend_layer_norm_workspace(n->rows, n->dim);
        if (need > 0 && (!n->workspace || !aligned_to(n->workspace, 16) || n->workspace_bytes < need))
            return fail(LEGEND_E_INVAL, "workspace must hold %lld bytes, aligned to 16", (long long)need);
        written.push_back(bytes_at(n->dweight, (int64_t)n->dim * ds));
        written.push_back(bytes_at(n->dbias, (int64_t)n->dim * ds));
        written.push_back(bytes_at(n->workspace, need));
        a.partial = static_cast<float*>(n->workspace);
        a.parts = norm_parts(n->rows, n->dim);
        a.dweight = n->dweight;
        a.dbias = n->dbias;
        a.dweight_type = n->dweight_type;
        a.accumulate = n->accumulate;
    }
    bool bad = false;
    if (n->rows > 0) {
        if (n->table >= 0) written.push_back(bytes_at(n->status, 4));
        if (!n->mean || !n->rstd) return fail(LEGEND_E_INVAL, "mean and rstd of the forward pass must not be NULL");
        Matrix x{}, dy{}, dx{};
        if (n->table < 0) {
            rc = check_matrix("x", n->x, n->x_stride, n->x_type, n->rows, n->dim, true, &x);
            if (rc) return rc;
        }
        rc = check_matrix("dy", n->dy, n->dy_stride, n->dy_type, n->rows, n->dim, true, &dy);
        if (rc) return rc;
        read.push_back(bytes_at(n->mean, n->rows * 4));
        read.push_back(bytes_at(n->rstd, n->rows * 4));
        if (n->dx) {
            rc = check_matrix("dx", n->dx, n->dx_stride, n->x_type, n->rows, n->dim, false, &dx);
            if (rc) return rc;
            bad = (n->table < 0 && meets(dx.range, x.range) && !same_place(x, dx)) || (meets(dx.range, dy.range) && !same_place(dx, dy));
            bad = bad || clash({dx.range}, written);
            bad = bad || clash({dx.range}, read);
        }
        bad = bad || clash(written, {x.range, dy.range});
        std::vector<Range> shared;
        read_ranges(n, &shared);
        if (n->dx) bad = bad || clash({dx.range}, shared);
        read.insert(read.end(), shared.begin(), shared.end());
        a.dy = n->dy;
        a.dy_stride = n->dy_stride;
        a.dy_type = n->dy_type;
        a.dx = n->dx;
        a.dx_stride = n->dx_stride;
    }
    if (bad || clash(written, read)) return fail(LEGEND_E_INVAL, "an output overlaps other memory of the call");
    if (n->table >= 0 && n->rows > 0) {
        bool rec = false;
        rc = recording(c, v.stream, &rec);
        if (rc) return rc;
        rc = ctx_tables_current(c, rec);
        if (rc) return rc;
    }
    DENSE_TRY(c, launch_norm_backward(v.stream, a));
    return LEGEND_OK;
    });
}

int legend_adamw_create(legend_ctx* c, const legend_adamw_config* cfg, const legend_adamw_tensor* tensors, int64_t n, legend_adamw** out) {
    return guarded("legend_adamw_create", [&]() -> int {
    if (out) *out = nullptr;
    DeviceScope scope;
    CtxView v;
    int rc = ctx_enter(c, &v);
    if (rc) return rc;
    if (!cfg || !tensors || !out) return fail(LEGEND_E_INVAL, "NULL argument");
    if (cfg->struct_size != sizeof(legend_adamw_config)) return fail(LEGEND_E_INVAL, "legend_adamw_config.struct_size mismatch");
    if (cfg->reserved != 0) return fail(LEGEND_E_INVAL, "reserved must be 0");
    if (n < 1 || n > (1 << 24)) return fail(LEGEND_E_INVAL, "n must be in [1, 2^24]");
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return fail(LEGEND_E_INVAL, "beta1 and beta2 must be in [0, 1)");
    if (!(cfg->eps >= 1e-15) || !(cfg->eps <= 1e15)) return fail(LEGEND_E_INVAL, "eps must be in [1e-15, 1e15]");
    if (!(cfg->max_norm >= 0.0) || !std::isfinite(cfg->max_norm)) return fail(LEGEND_E_INVAL, "max_norm must be finite and not negative");
    std::vector<const void*> grads((size_t)n);
    int64_t total = 0, total_bytes = 0;
    int32_t kinds = 0;
    for (int64_t k = 0; k < n; ++k) {
        rc = check_tensor(tensors[k], k);
        if (rc) return rc;
        grads[(size_t)k] = tensors[k].grad;
        total += tensors[k].count;
        total_bytes += tensor_bytes(tensors[k]);
        kinds |= tensors[k].state_type == LEGEND_STATE_BLOCK ? 2 : 1;
        if (total > ((int64_t)1 << 48)) return fail(LEGEND_E_INVAL, "too many elements");
    }
    struct Holder {
        legend_adamw* o;
        ~Holder() {
            if (!o) return;
            if (o->mem) (void)hipFree(o->mem);
            delete o;
        }
    } hold{new legend_adamw};
    legend_adamw* o = hold.o;
    o->device = v.device;
    o->cfg = *cfg;
    o->tensors.assign(tensors, tensors + n);
    rc = check_apart(o->tensors, grads.data(), &o->used);
    if (rc) return rc;
    rc = refuse_recording(c, v.stream, "an optimiser cannot be created");
    if (rc) return rc;

    o->unit_elems = adam_unit_elems(total);
    o->stream = total_bytes > kStreamBytes;
    o->kinds = kinds;
    std::vector<AdamTensor> desc((size_t)n);
    for (int64_t k = 0; k < n; ++k) {
        const legend_adamw_tensor& t = tensors[k];
        desc[(size_t)k] = AdamTensor{t.param, t.master, t.m, t.v, t.m_scale, t.v_scale, t.count, o->units, t.weight_decay, t.lr_scale,
                                     t.param_type, t.grad_type, t.state_type, (int32_t)k};
        o->units += (t.count + o->unit_elems - 1) / o->unit_elems;
    }
    if (o->units > (1 << 28)) return fail(LEGEND_E_INVAL, "too many elements");
    std::vector<int32_t> unit_tensor((size_t)o->units);
    for (int64_t k = 0, u = 0; k < n; ++k)
        for (int64_t left = tensors[k].count; left > 0; left -= o->unit_elems) unit_tensor[(size_t)u++] = (int32_t)k;

    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    const size_t b_state = up(sizeof(AdamState)), b_partial = up(sizeof(double) * kAdamNormParts), b_desc = up(sizeof(AdamTensor) * (size_t)n),
                 b_grads = up(sizeof(void*) * (size_t)n), b_units = up(sizeof(int32_t) * (size_t)std::max<int64_t>(o->units, 1));
    if (hipMalloc((void**)&o->mem, b_state + b_partial + b_desc + b_grads + b_units) != hipSuccess) {
        (void)hipGetLastError();
        o->mem = nullptr;
        return fail(LEGEND_E_NOMEM, "device allocation of the optimiser's tables failed");
    }
    char* p = o->mem;
    o->d_state = reinterpret_cast<AdamState*>(p); p += b_state;
    o->d_partial = reinterpret_cast<double*>(p); p += b_partial;
    o->d_tensors = reinterpret_cast<AdamTensor*>(p); p += b_desc;
    o->d_grads = reinterpret_cast<const void**>(p); p += b_grads;
    o->d_unit_tensor = reinterpret_cast<int32_t*>(p);
    AdamState s;
    adam_state_at(&s, 0, cfg->beta1, cfg->beta2);
    DENSE_TRY(c, hipMemcpyAsync(o->d_state, &s, sizeof s, hipMemcpyHostToDevice, v.stream));
    DENSE_TRY(c, hipMemcpyAsync(o->d_tensors, desc.data(), sizeof(AdamTensor) * (size_t)n, hipMemcpyHostToDevice, v.stream));
    DENSE_TRY(c, hipMemcpyAsync(o->d_grads, grads.data(), sizeof(void*) * (size_t)n, hipMemcpyHostToDevice, v.stream));
    if (o->units > 0)
        DENSE_TRY(c, hipMemcpyAsync(o->d_unit_tensor, unit_tensor.data(), sizeof(int32_t) * (size_t)o->units, hipMemcpyHostToDevice, v.stream));
    DENSE_TRY(c, hipStreamSynchronize(v.stream));
    ctx_keep(c, o, true);
    o->ctx = c;
    hold.o = nullptr;
    *out = o;
    return LEGEND_OK;
    });
}

int legend_adamw_destroy(legend_adamw* o) {
    return guarded("legend_adamw_destroy", [&]() -> int {
    if (!o) return LEGEND_OK;
    DeviceScope scope;
    (void)hipSetDevice(o->device);
    CtxView v;
    if (o->ctx) {
        if (ctx_enter(o->ctx, &v) == LEGEND_OK) {
            int rc = refuse_recording(o->ctx, v.stream, "an optimiser cannot be destroyed");
            if (rc == LEGEND_E_STATE) return rc;
            (void)hipStreamSynchronize(v.stream);
        }
        ctx_keep(o->ctx, o, false);
    }
    if (o->mem) (void)hipFree(o->mem);
    delete o;
    return LEGEND_OK;
    });
}

int legend_adamw_step(legend_adamw* o, double lr, const float* lr_factor, const float* grad_scale, float* norm) {
    return guarded("legend_adamw_step", [&]() -> int {
    DeviceScope scope;
    CtxView v;
    int rc = enter_opt(o, &v);
    if (rc) return rc;
    if (!(lr >= 0.0) || !std::isfinite(lr)) return fail(LEGEND_E_INVAL, "lr must be finite and not negative");
    if (!aligned_to(lr_factor, 4) || !aligned_to(grad_scale, 4) || !aligned_to(norm, 4)) return fail(LEGEND_E_INVAL, "a scalar is not aligned to its type");
    if (lies_in(o->used, lr_factor) || lies_in(o->used, grad_scale) || lies_in(o->used, norm) || (norm && (norm == lr_factor || norm == grad_scale)))
        return fail(LEGEND_E_INVAL, "lr_factor, grad_scale or norm lies in other memory of the step");
    AdamParams a{};
    a.tensors = o->d_tensors;
    a.grads = o->d_grads;
    a.unit_tensor = o->d_unit_tensor;
    a.units = o->units;
    a.unit_elems = o->unit_elems;
    a.state = o->d_state;
    a.partial = o->d_partial;
    a.grad_scale = grad_scale;
    a.lr_factor = lr_factor;
    a.norm_out = norm;
    a.lr = lr;
    a.beta1 = o->cfg.beta1;
    a.beta2 = o->cfg.beta2;
    a.eps = o->cfg.eps;
    a.max_norm = o->cfg.max_norm;
    a.seed = o->cfg.seed;
    a.stream = o->stream ? 1 : 0;
    a.kinds = o->kinds;
    a.with_norm = o->cfg.max_norm > 0.0 || norm ? 1 : 0;
    DENSE_TRY(o->ctx, launch_adamw(v.stream, a));
    return LEGEND_OK;
    });
}

int legend_adamw_set_gradients(legend_adamw* o, const void* const* grads, int64_t n) {
    return guarded("legend_adamw_set_gradients", [&]() -> int {
    DeviceScope scope;
    CtxView v;
    int rc = enter_opt(o, &v);
    if (rc) return rc;
    if (!grads) return fail(LEGEND_E_INVAL, "NULL argument");
    if (n != (int64_t)o->tensors.size()) return fail(LEGEND_E_INVAL, "%lld gradients for %lld tensors", (long long)n, (long long)o->tensors.size());
    for (int64_t k = 0; k < n; ++k) {
        const legend_adamw_tensor& t = o->tensors[(size_t)k];
        if (t.count > 0 && (!grads[k] || !aligned_to(grads[k], type_size(t.grad_type))))
            return fail(LEGEND_E_INVAL, "gradient %lld is NULL or not aligned to its elements", (long long)k);
    }
    std::vector<std::pair<uintptr_t, uintptr_t>> used;
    rc = check_apart(o->tensors, grads, &used);
    if (rc) return rc;
    rc = refuse_recording(o->ctx, v.stream, "gradients cannot be set");
    if (rc) return rc;
    DENSE_TRY(o->ctx, hipMemcpyAsync(o->d_grads, grads, sizeof(void*) * (size_t)n, hipMemcpyHostToDevice, v.stream));
    DENSE_TRY(o->ctx, hipStreamSynchronize(v.stream));
    o->used.swap(used);
    return LEGEND_OK;
    });
}

int legend_adamw_get_steps(legend_adamw* o, int64_t* steps, int64_t* skipped) {
    return guarded("legend_adamw_get_steps", [&]() -> int {
    DeviceScope scope;
    CtxView v;
    int rc = enter_opt(o, &v);
    if (rc) return rc;
    rc = refuse_recording(o->ctx, v.stream, "steps cannot be read");
    if (rc) return rc;
    AdamState s;
    DENSE_TRY(o->ctx, hipMemcpyAsync(&s, o->d_state, sizeof s, hipMemcpyDeviceToHost, v.stream));
    DENSE_TRY(o->ctx, hipStreamSynchronize(v.stream));
    if (steps) *steps = s.steps;
    if (skipped) *skipped = s.skipped;
    return LEGEND_OK;
    });
}

int legend_adamw_set_steps(legend_adamw* o, int64_t steps) {
    return guarded("legend_adamw_set_steps", [&]() -> int {
    DeviceScope scope;
    CtxView v;
    int rc = enter_opt(o, &v);
    if (rc) return rc;
    if (steps < 0 || steps > ((int64_t)1 << 48)) return fail(LEGEND_E_INVAL, "steps out of range");
    rc = refuse_recording(o->ctx, v.stream, "steps cannot be set");
    if (rc) return rc;
    AdamState s;
    adam_state_at(&s, steps, o->cfg.beta1, o->cfg.beta2);
    DENSE_TRY(o->ctx, hipMemcpyAsync(o->d_state, &s, sizeof s, hipMemcpyHostToDevice, v.stream));
    DENSE_TRY(o->ctx, hipStreamSynchronize(v.stream));
    return LEGEND_OK;
    });
}

}  // extern "C"
