// Layer norm over rows of a matrix or of a resident table: forward, and backward with the sums over rows that the weight's
// and the bias's gradients are.
//
//   mean = sum x / d,  c = x - mean,  var = sum c^2 / d,  rstd = 1 / sqrt(var + eps),  xh = c rstd,  y = xh w + b
//   u = dy w,  dx = rstd (u - mean(u) - xh mean(u xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// All arithmetic is fp32 from the loaded values to the one rounding of what is stored.  The variance is a second sum, of
// squares of what is left of the mean: sum x^2 - d mean^2 would lose the digits that an offset common to a row takes up.
// What the rounding of the mean to fp32 leaves, left = sum c / d, is taken off in the same sweep: var = sum c^2 / d - left^2,
// and by a third sum where left^2 is more than kLeftShare of the first term (rows whose spread is lost in their offset).
#include "legend_internal.h"
#include "device_utils.h"
#include "tensor_types.h"

namespace legend {

constexpr float kLeftShare = 9.765625e-4f;   // 2^-10: the difference then loses a thousandth of a bit

// Address of row r, or null (and its bit in *status) for a row of a table that the call may not read.
template <class XT>
__device__ inline const XT* source_row(const NormParams& a, int64_t r, bool reports) {
    if (!a.status) return static_cast<const XT*>(a.x) + r * a.x_stride;
    const int64_t id = a.ids ? a.ids[r] : r;
    if (id < 0 || id >= a.table_rows) {
        if (reports) atomicOr(a.status, 1u);
        return nullptr;
    }
    if (a.rel_base) return reinterpret_cast<const XT*>(a.rel_base + id * a.dim);
    const int64_t p = id / a.rows_per_partition;
    const float* base = a.part_base[p];
    if (!base) {
        if (reports) atomicOr(a.status, 2u);
        return nullptr;
    }
    return reinterpret_cast<const XT*>(base + (id - p * a.rows_per_partition) * a.dim);
}

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int k = 1; k < kWave; k <<= 1) v += wave_shfl_xor(v, k);
    return v;
}

// Sums of two numbers over a workgroup, in every thread; `box` holds 2 x 16 floats.  Ends with every wave past its reads.
__device__ inline void block_sum2(float& p, float& q, float* box) {
    p = wave_sum(p);
    q = wave_sum(q);
    const int waves = blockDim.x / kWave, w = threadIdx.x / kWave;
    if (lane_id() == 0) { box[w] = p; box[16 + w] = q; }
    __syncthreads();
    p = q = 0.f;
    for (int k = 0; k < waves; ++k) { p += box[k]; q += box[16 + k]; }
    __syncthreads();
}

// ---- rows of any length: a workgroup a row, which it reads again for every sweep --------------------------------------

template <class XT, class YT>
__global__ void __launch_bounds__(1024) k_norm_forward_long(NormParams a) {
    __shared__ float box[32];
    const int d = a.dim;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const XT* x = source_row<XT>(a, r, threadIdx.x == 0);
        YT* y = static_cast<YT*>(a.y) + r * a.y_stride;
        float mean = 0.f, rstd = 0.f, left = 0.f, none = 0.f;
        if (x) {
            for (int c = threadIdx.x; c < d; c += blockDim.x) mean += (float)x[c];
            block_sum2(mean, none, box);
            mean /= (float)d;
            float sq = 0.f;
            for (int c = threadIdx.x; c < d; c += blockDim.x) {
                const float v = (float)x[c] - mean;
                left += v;
                sq += v * v;
            }
            block_sum2(left, sq, box);
            left /= (float)d;
            float var = sq / (float)d;
            if (left * left > kLeftShare * var) {
                sq = 0.f;
                for (int c = threadIdx.x; c < d; c += blockDim.x) {
                    const float v = (float)x[c] - mean - left;
                    sq += v * v;
                }
                block_sum2(sq, none, box);
                var = sq / (float)d;
            } else {
                var -= left * left;
            }
            rstd = 1.0f / sqrtf(var + a.eps);
            for (int c = threadIdx.x; c < d; c += blockDim.x) {
                float v = ((float)x[c] - mean - left) * rstd;
                if (a.weight) v *= load_as(a.weight, c, a.weight_type);
                if (a.bias) v += load_as(a.bias, c, a.weight_type);
                y[c] = (YT)v;
            }
        } else {
            for (int c = threadIdx.x; c < d; c += blockDim.x) y[c] = (YT)0.f;
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mean + left;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <class XT, class YT>
__global__ void __launch_bounds__(1024) k_norm_backward_long(NormParams a) {
    __shared__ float box[32];
    const int d = a.dim;
    float* pw = a.partial + (int64_t)blockIdx.x * 2 * d;       // sums of this workgroup's rows
    float* pb = pw + d;
    bool first = true;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const XT* x = source_row<XT>(a, r, threadIdx.x == 0);
        const YT* dy = static_cast<const YT*>(a.dy) + r * a.dy_stride;
        XT* dx = a.dx ? static_cast<XT*>(a.dx) + r * a.dx_stride : nullptr;
        if (!x) {
            if (dx) for (int c = threadIdx.x; c < d; c += blockDim.x) dx[c] = (XT)0.f;
            continue;
        }
        const float mean = a.mean[r], rstd = a.rstd[r];
        float su = 0.f, sx = 0.f;
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            const float g = (float)dy[c], xh = ((float)x[c] - mean) * rstd;
            const float u = a.weight ? g * load_as(a.weight, c, a.weight_type) : g;
            su += u;
            sx += u * xh;
            if (a.partial) {
                pw[c] = first ? g * xh : pw[c] + g * xh;
                pb[c] = first ? g : pb[c] + g;
            }
        }
        first = false;
        if (!dx) continue;
        block_sum2(su, sx, box);
        su /= (float)d;
        sx /= (float)d;
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            const float g = (float)dy[c], xh = ((float)x[c] - mean) * rstd;
            const float u = a.weight ? g * load_as(a.weight, c, a.weight_type) : g;
            dx[c] = (XT)(rstd * (u - su - xh * sx));
        }
    }
    if (a.partial && first)
        for (int c = threadIdx.x; c < d; c += blockDim.x) pw[c] = pb[c] = 0.f;
}

// Sums of the workgroups' partial sums, in 64 bits and in a fixed order.
__global__ void __launch_bounds__(256) k_norm_sums(NormParams a) {
    const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= 2 * (int64_t)a.dim) return;
    void* out = c < a.dim ? a.dweight : a.dbias;
    if (!out) return;
    const int64_t at = c < a.dim ? c : c - a.dim;
    double s = a.accumulate ? (double)load_as(out, at, a.dweight_type) : 0.0;
    for (int p = 0; p < a.parts; ++p) s += (double)a.partial[(int64_t)p * 2 * a.dim + c];
    store_as(out, at, a.dweight_type, (float)s);
}

// ---- launches ------------------------------------------------------------------------------------------------------

int norm_parts(int64_t rows, int32_t dim) {
    (void)dim;
    return (int)(rows < 512 ? rows : 512);
}

template <class F>
static hipError_t for_types(int x_type, int y_type, F&& f) {
    if (x_type == LEGEND_TYPE_FLOAT) {
        if (y_type == LEGEND_TYPE_FLOAT) return f(float{}, float{});
        if (y_type == LEGEND_TYPE_BFLOAT) return f(float{}, bf16_t{});
        return f(float{}, half_t{});
    }
    if (x_type == LEGEND_TYPE_BFLOAT) return y_type == LEGEND_TYPE_FLOAT ? f(bf16_t{}, float{}) : f(bf16_t{}, bf16_t{});
    return y_type == LEGEND_TYPE_FLOAT ? f(half_t{}, float{}) : f(half_t{}, half_t{});
}

hipError_t launch_norm_forward(hipStream_t st, const NormParams& a) {
    if (a.rows <= 0) return hipSuccess;
    return for_types(a.x_type, a.y_type, [&](auto xt, auto yt) {
        const unsigned grid = (unsigned)(a.rows < 65536 ? a.rows : 65536);
        k_norm_forward_long<decltype(xt), decltype(yt)><<<grid, 256, 0, st>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_norm_backward(hipStream_t st, const NormParams& a) {
    if (a.rows > 0) {
        hipError_t e = for_types(a.x_type, a.dy_type, [&](auto xt, auto yt) {
            const unsigned grid = a.partial ? (unsigned)a.parts : (unsigned)(a.rows < 65536 ? a.rows : 65536);
            k_norm_backward_long<decltype(xt), decltype(yt)><<<grid, 256, 0, st>>>(a);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    if (!a.dweight && !a.dbias) return hipSuccess;
    const unsigned grid = (unsigned)((2 * (int64_t)a.dim + 255) / 256);
    k_norm_sums<<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace legend
