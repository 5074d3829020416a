// Layer norm over rows of a matrix or of a resident table, forward.
//
//   mean = sum x / d,  c = x - mean,  var = sum c^2 / d,  rstd = 1 / sqrt(var + eps),  xh = c rstd,  y = xh w + b
//
// All arithmetic is fp32 from the loaded values to the one rounding of what is stored.  The variance is a second sum, of
// squares of what is left of the mean: sum x^2 - d mean^2 would lose the digits that an offset common to a row takes up.
// What the rounding of the mean to fp32 leaves, left = sum c / d, is taken off in the same sweep: var = sum c^2 / d - left^2,
// and by a third sum where left^2 is more than kLeftShare of the first term (rows whose spread is lost in their offset).  Where the squares
// leave fp32, the third sum is of squares in units of 2^192.
//
// A row stays in the registers of 8 to 512 threads from its one read to its one write; weight and bias stay there from row to row,
// and the next row's loads are on their way while a row is worked on.  Bound by HBM: an element is read and written once, for some
// ten vector instructions.  16384 x 4096 bf16: 51 us, 5.3 TB/s (a workgroup a row that reads it again for every sweep: 267 us; without the
// loads ahead and with a branch at each of them: 86); 50 000 x 100 table rows to bf16: 10.3 us, of which 2.5 are a launch's.
#include "norm_rows.h"

#include <type_traits>

namespace legend {

// Of squares that leave fp32, the difference from themselves is NaN, otherwise 0: no constant to compare with.  (A compare with infinity takes an
// 81st scalar register, with which a compute unit holds 28 waves instead of 32: 50 000 x 100 table rows 11.8 against 10.6 us.)
constexpr float kSmallUnit = 0x1p-96f;            // sums of 2^20 squares of anything below 3e38 stay within fp32
// 1 / sqrt(variance + eps) from the variance of a row that was multiplied by `unit`, a power of two.
__device__ inline float row_rstd(float var, float eps, float unit) { return 1.f / sqrtf(var + eps * unit * unit) * unit; }

// Waves of a SIMD at most.  Of rows of 2049 to 4096 columns four workgroups a compute unit, so that the grid's eight are two whole rounds: five, which
// the registers would allow, make the second one a short one (16384 x 4096 bf16 54 against 52.5 us).
template <class S>
constexpr int waves_at_most() { return S::NE == 16 && S::T == 256 ? 4 : 8; }

template <class XT, class YT, class S, bool TABLE>
__global__ void __launch_bounds__(S::threads) __attribute__((amdgpu_waves_per_eu(1, waves_at_most<S>()))) k_norm_forward(NormParams a) {
    constexpr int NE = S::NE, T = S::T, R = S::R;
    __shared__ float box[2][32];
    int turn = 0;
    const int d = a.dim, lane = threadIdx.x % T;
    const float inv_d = 1.f / (float)d;
    const int64_t stride = (int64_t)gridDim.x * S::groups * R;
    RowColumns<XT, S> next[R];
    bool next_good[R];
    RowSource<XT, TABLE, R> source;
    auto load = [&](int64_t r0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const XT* src = source.row(a, r0, i, lane == 0);
            next_good[i] = src != nullptr;
            if (src) next[i].load(src, d, lane);
            else next[i].clear();
        }
    };
    int64_t r0 = ((int64_t)blockIdx.x * S::groups + threadIdx.x / T) * R;
    source.name(a, r0);
    load(r0);
    source.name(a, r0 + stride);
    float w[NE], b[NE];
    load_parameter<S>(a.weight, a.weight_type, 1.f, d, lane, w);
    load_parameter<S>(a.bias, a.weight_type, 0.f, d, lane, b);
    for (; r0 < a.rows; r0 += stride) {
        float x[R][NE];
        bool good[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            good[i] = next_good[i];
#pragma unroll
            for (int k = 0; k < NE; ++k) x[i][k] = S::inside(k, lane, d) ? next[i].number(k) : 0.f;
        }
        if (r0 + stride < a.rows) {                            // the next rows arrive while these are worked on
            load(r0 + stride);
            source.name(a, r0 + 2 * stride);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (r0 + i >= a.rows) continue;
            float sum = 0.f, none = 0.f;
#pragma unroll
            for (int k = 0; k < NE; ++k) sum += x[i][k];
            row_sum<T, 1>(sum, none, box, turn);
            const float mean = sum * inv_d;
            float left = 0.f, sq = 0.f;
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                x[i][k] = S::inside(k, lane, d) ? x[i][k] - mean : 0.f;
                left += x[i][k];
                sq = fmaf(x[i][k], x[i][k], sq);
            }
            row_sum<T, 2>(left, sq, box, turn);
            left *= inv_d;
            float var = sq * inv_d, unit = 1.f;
            const float beyond = sq - sq;
            if (!(left * left + beyond <= kLeftShare * var)) {
                unit = beyond == 0.f ? 1.f : kSmallUnit;
                sq = 0.f;
#pragma unroll
                for (int k = 0; k < NE; ++k) {
                    const float v = S::inside(k, lane, d) ? (x[i][k] - left) * unit : 0.f;
                    sq = fmaf(v, v, sq);
                }
                row_sum<T, 1>(sq, none, box, turn);
                var = sq * inv_d;
            } else {
                var = fmaf(-left, left, var);
            }
            const float rstd = good[i] ? row_rstd(var, a.eps, unit) : 0.f;
#pragma unroll
            for (int k = 0; k < NE; ++k) x[i][k] = good[i] ? fmaf((x[i][k] - left) * rstd, w[k], b[k]) : 0.f;
            store_columns<S>(static_cast<YT*>(a.y) + (r0 + i) * a.y_stride, d, lane, x[i]);
            if (lane == 0) {
                if (a.mean) a.mean[r0 + i] = good[i] ? mean + left : 0.f;
                if (a.rstd) a.rstd[r0 + i] = rstd;
            }
        }
    }
}

// ---- rows that do not fit a workgroup's registers: 16384 columns at a time, read again for every sweep ----------------

template <class XT, class YT, NormColumns Q>
__global__ void __launch_bounds__(1024) k_norm_forward_long(NormParams a) {
    typedef NormShape<16, 1024, 1, 0, Q, 1024> S;
    constexpr int NE = S::NE, PANEL = S::NE * S::T;
    __shared__ float box[2][32];
    int turn = 0;
    const int d = a.dim, lane = threadIdx.x;
    const float inv_d = 1.f / (float)d;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const XT* x = static_cast<const XT*>(a.x) + r * a.x_stride;
        YT* y = static_cast<YT*>(a.y) + r * a.y_stride;
        float mean = 0.f, rstd = 0.f, left = 0.f, none = 0.f;
        float v[NE];
        // f(first column, columns left): `v` holds the panel's numbers less `shift`, zeros behind the row's end
        auto sweep = [&](float shift, auto&& f) {
            for (int at = 0; at < d; at += PANEL) {
                RowColumns<XT, S> p;
                p.load(x + at, d - at, lane);
#pragma unroll
                for (int k = 0; k < NE; ++k) v[k] = S::inside(k, lane, d - at) ? p.number(k) - shift : 0.f;
                f(at, d - at);
            }
        };
        sweep(0.f, [&](int, int) {
#pragma unroll
            for (int k = 0; k < NE; ++k) mean += v[k];
        });
        row_sum<1024, 1>(mean, none, box, turn);
        mean *= inv_d;
        float sq = 0.f;
        sweep(mean, [&](int, int) {
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                left += v[k];
                sq = fmaf(v[k], v[k], sq);
            }
        });
        row_sum<1024, 2>(left, sq, box, turn);
        left *= inv_d;
        float var = sq * inv_d, unit = 1.f;
        const float beyond = sq - sq;
        if (!(left * left + beyond <= kLeftShare * var)) {
            unit = beyond == 0.f ? 1.f : kSmallUnit;
            sq = 0.f;
            sweep(mean, [&](int, int n) {
#pragma unroll
                for (int k = 0; k < NE; ++k) {
                    const float c = S::inside(k, lane, n) ? (v[k] - left) * unit : 0.f;
                    sq = fmaf(c, c, sq);
                }
            });
            row_sum<1024, 1>(sq, none, box, turn);
            var = sq * inv_d;
        } else {
            var = fmaf(-left, left, var);
        }
        rstd = row_rstd(var, a.eps, unit);
        sweep(mean, [&](int at, int n) {
            float w[NE], b[NE];
            load_parameter<S>(a.weight, a.weight_type, 1.f, n, lane, w, at);
            load_parameter<S>(a.bias, a.weight_type, 0.f, n, lane, b, at);
#pragma unroll
            for (int k = 0; k < NE; ++k) v[k] = fmaf((v[k] - left) * rstd, w[k], b[k]);
            store_columns<S>(y + at, n, lane, v);
        });
        if (lane == 0) {
            if (a.mean) a.mean[r] = mean + left;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

hipError_t launch_norm_forward(hipStream_t st, const NormParams& a) {
    if (a.rows <= 0) return hipSuccess;
    if (a.status && a.dim > kTableRowMax) return hipErrorInvalidValue;
    return for_types(a.x_type, a.y_type, [&](auto xt, auto yt) {
        typedef decltype(xt) XT;
        typedef decltype(yt) YT;
        if (a.dim > kNormRowMax) {
            const unsigned grid = (unsigned)(a.rows < 512 ? a.rows : 512);
            if (a.dim % 4 == 0) k_norm_forward_long<XT, YT, QUADS><<<grid, 1024, 0, st>>>(a);
            else k_norm_forward_long<XT, YT, RAGGED><<<grid, 1024, 0, st>>>(a);
        } else {
            for_shape<1, 256>(a.dim, [&](auto s) {
                typedef decltype(s) S;
                // at most 2048 threads a compute unit, what it holds of the kernels with up to 64 registers and twice what it holds of those with
                // up to 128, so that weight and bias are loaded once for several rows (one row a workgroup: 63 against 51 us for 16384 x
                // 4096 bf16)
                const int64_t need = (a.rows + S::groups * S::R - 1) / (S::groups * S::R), most = 256 * 2048 / S::threads;
                const unsigned grid = (unsigned)(need < most ? need : most);
                if (!a.status) k_norm_forward<XT, YT, S, false><<<grid, S::threads, 0, st>>>(a);
                else if constexpr (std::is_same<XT, float>::value && S::LOW < kTableRowMax) k_norm_forward<XT, YT, S, true><<<grid, S::threads, 0, st>>>(a);
                return 0;
            });
        }
        return hipGetLastError();
    });
}

}  // namespace legend
