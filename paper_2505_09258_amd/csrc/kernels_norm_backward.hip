// Layer norm, backward: the gradient of the rows, and the sums over rows that the weight's and the bias's gradients are.
//
//   xh = (x - mean) rstd,  u = dy w,  dx = rstd (u - mean(u) - xh mean(u xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// A row's x and dy stay in the registers of 8 to 512 threads.  A thread keeps the same columns from row to row and adds up its
// columns' dw and db in fp32 (over rows / 512 rows from 1025 to 4096 columns, rows / 256 above, rows / 4096 and less below); a
// workgroup writes its sums once, and a second kernel adds those in 64 bits, in a fixed order (no atomics: the same bits every
// time).  Bound by HBM.  16384 x 4096 bf16: 78 us and 5 for the sums, 5.0 TB/s (first form 1072 us; without the next row's loads ahead
// 204); 50 000 x 100 table rows, sums only: 11 us and 4 (workgroups of 256 threads: 22 together).
#include "norm_rows.h"

#include <type_traits>

namespace legend {

// A column's sum over all rows (c < dim: of the weight's gradient) where the caller wants it.
__device__ inline void put_sum(const NormParams& a, int64_t c, double s) {
    void* out = c < a.dim ? a.dweight : a.dbias;
    if (!out) return;
    const int64_t at = c < a.dim ? c : c - a.dim;
    if (a.accumulate) s += (double)load_as(out, at, a.dweight_type);
    store_as(out, at, a.dweight_type, (float)s);
}

template <class XT, class YT, class S, bool TABLE>
__global__ void __launch_bounds__(S::threads) k_norm_backward(NormParams a) {
    constexpr int NE = S::NE, T = S::T, R = S::R, G = S::groups;
    // The weight and the columns' sums in registers; for the longest rows the weight is read again for every row (from L2) and the
    // sums lie in LDS (128 KB), each thread's in a place of its own.  (4099 x 16383 fp32: 173 us, with both in registers, which then do
    // not suffice, 216; 4096 x 16384 bf16: 92 and 105.)
    constexpr bool KEEP = NE < 32;
    __shared__ float box[2][32];
    __shared__ __align__(16) float sums[G > 1 || !KEEP ? 2 * S::threads * NE : 4];
    int turn = 0;
    const int d = a.dim, lane = threadIdx.x % T;
    const float inv_d = 1.f / (float)d;
    const int64_t stride = (int64_t)gridDim.x * G * R;
    RowColumns<XT, S> next_x[R];
    RowColumns<YT, S> next_g[R];
    float next_mean[R], next_rstd[R];
    bool next_good[R];                           // a table's row that may be read
    RowSource<XT, TABLE, R> source;
    auto load = [&](int64_t r0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const XT* src = source.row(a, r0, i, lane == 0);
            next_mean[i] = next_rstd[i] = 0.f;
            next_good[i] = src != nullptr;
            if (src) {
                next_x[i].load(src, d, lane);
                next_g[i].load(static_cast<const YT*>(a.dy) + (r0 + i) * a.dy_stride, d, lane);
                next_mean[i] = a.mean[r0 + i];
                next_rstd[i] = a.rstd[r0 + i];
            } else {                             // nothing to add, a gradient of zeros
                next_x[i].clear();
                next_g[i].clear();
            }
        }
    };
    int64_t r0 = ((int64_t)blockIdx.x * G + threadIdx.x / T) * R;
    source.name(a, r0);
    load(r0);
    source.name(a, r0 + stride);
    float w[NE], dw[KEEP ? NE : 1], db[KEEP ? NE : 1];
    float4* far_w = reinterpret_cast<float4*>(sums) + threadIdx.x;             // !KEEP: this thread's sums, S::threads apart
    float4* far_b = far_w + S::threads * (NE / 4);
    if (KEEP) load_parameter<S>(a.weight, a.weight_type, 1.f, d, lane, w);
#pragma unroll
    for (int k = 0; k < NE; ++k) {
        if (KEEP) dw[k] = db[k] = 0.f;
        else if (k % 4 == 0) far_w[k / 4 * S::threads] = far_b[k / 4 * S::threads] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (; r0 < a.rows; r0 += stride) {
        float x[R][NE], g[R][NE], rstd[R];
        bool good[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rstd[i] = next_rstd[i];
            good[i] = !TABLE || next_good[i];
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                // (an access behind the row's end holds the row's last columns: what their zero gradients meet is of no account)
                x[i][k] = (next_x[i].number(k) - next_mean[i]) * rstd[i];
                g[i][k] = S::inside(k, lane, d) ? next_g[i].number(k) : 0.f;
            }
        }
        if (!KEEP) load_parameter<S>(a.weight, a.weight_type, 1.f, d, lane, w);
        if (r0 + stride < a.rows) {                            // the next rows arrive while these are worked on
            load(r0 + stride);
            source.name(a, r0 + 2 * stride);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (r0 + i >= a.rows) continue;
            float su = 0.f, sx = 0.f;
            if (!KEEP && a.partial) {
#pragma unroll
                for (int k = 0; k < NE; k += 4) {
                    float4 p = far_w[k / 4 * S::threads], q = far_b[k / 4 * S::threads];
                    p.x = fmaf(g[i][k], x[i][k], p.x);
                    p.y = fmaf(g[i][k + 1], x[i][k + 1], p.y);
                    p.z = fmaf(g[i][k + 2], x[i][k + 2], p.z);
                    p.w = fmaf(g[i][k + 3], x[i][k + 3], p.w);
                    q.x += g[i][k]; q.y += g[i][k + 1]; q.z += g[i][k + 2]; q.w += g[i][k + 3];
                    far_w[k / 4 * S::threads] = p;
                    far_b[k / 4 * S::threads] = q;
                }
            }
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                if (KEEP) {
                    dw[k] = fmaf(g[i][k], x[i][k], dw[k]);
                    db[k] += g[i][k];
                }
                g[i][k] *= w[k];
                su += g[i][k];
                sx = fmaf(g[i][k], x[i][k], sx);
            }
            if (!a.dx) continue;
            row_sum<T, 2>(su, sx, box, turn);
            su *= inv_d;
            sx *= inv_d;
#pragma unroll
            for (int k = 0; k < NE; ++k) g[i][k] = good[i] ? rstd[i] * fmaf(-x[i][k], sx, g[i][k] - su) : 0.f;   // (a weight need not be finite)
            store_columns<S>(static_cast<XT*>(a.dx) + (r0 + i) * a.dx_stride, d, lane, g[i]);
        }
    }
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * d;
    if (!KEEP) {
        float t[NE];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int k = 0; k < NE; k += 4) *reinterpret_cast<float4*>(t + k) = (half ? far_b : far_w)[k / 4 * S::threads];
            store_columns<S>(out + half * d, d, lane, t);
        }
        return;
    }
    if (G == 1) {
        store_columns<S>(out, d, lane, dw);
        store_columns<S>(out + d, d, lane, db);
        return;
    }
    float* mine = sums + (threadIdx.x / T) * (2 * T * NE);
#pragma unroll
    for (int k = 0; k < NE; ++k) {
        if (!S::inside(k, lane, d)) continue;
        mine[S::column(k, lane, d)] = dw[KEEP ? k : 0];
        mine[T * NE + S::column(k, lane, d)] = db[KEEP ? k : 0];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * T * NE; c += S::threads) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < G; ++k) s += sums[k * (2 * T * NE) + c];
        const int col = c < T * NE ? c : c - T * NE;
        if (col >= d) continue;
        if (a.parts == 1) put_sum(a, c < T * NE ? col : d + col, (double)s);
        else out[c < T * NE ? col : d + col] = s;
    }
}

// ---- rows that do not fit a workgroup's registers: 16384 columns at a time ---------------------------------------------

template <class XT, class YT, NormColumns Q>
__global__ void __launch_bounds__(1024) k_norm_backward_long(NormParams a) {
    typedef NormShape<16, 1024, 1, 0, Q, 1024> S;
    constexpr int NE = S::NE, PANEL = S::NE * S::T;
    __shared__ float box[2][32];
    int turn = 0;
    const int d = a.dim, lane = threadIdx.x;
    const float inv_d = 1.f / (float)d;
    float* pw = a.partial + (int64_t)blockIdx.x * 2 * d;       // sums of this workgroup's rows
    float* pb = pw + d;
    bool first = true;
    float xh[NE], g[NE], w[NE];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const XT* x = static_cast<const XT*>(a.x) + r * a.x_stride;
        const YT* dy = static_cast<const YT*>(a.dy) + r * a.dy_stride;
        XT* dx = a.dx ? static_cast<XT*>(a.dx) + r * a.dx_stride : nullptr;
        const float mean = a.mean[r], rstd = a.rstd[r];
        auto take = [&](int at) {
            RowColumns<XT, S> px;
            RowColumns<YT, S> pg;
            px.load(x + at, d - at, lane);
            pg.load(dy + at, d - at, lane);
            load_parameter<S>(a.weight, a.weight_type, 1.f, d - at, lane, w, at);
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                xh[k] = (px.number(k) - mean) * rstd;
                g[k] = S::inside(k, lane, d - at) ? pg.number(k) : 0.f;
            }
        };
        float su = 0.f, sx = 0.f;
        for (int at = 0; at < d; at += PANEL) {
            take(at);
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                const float u = g[k] * w[k];
                su += u;
                sx = fmaf(u, xh[k], sx);
            }
            if (!a.partial) continue;
            RowColumns<float, S> pw_old, pb_old;
            if (first) {
                pw_old.clear();
                pb_old.clear();
            } else {
                pw_old.load(pw + at, d - at, lane);
                pb_old.load(pb + at, d - at, lane);
            }
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                xh[k] = fmaf(g[k], xh[k], pw_old.number(k));
                g[k] += pb_old.number(k);
            }
            store_columns<S>(pw + at, d - at, lane, xh);
            store_columns<S>(pb + at, d - at, lane, g);
        }
        first = false;
        if (!dx) continue;
        row_sum<1024, 2>(su, sx, box, turn);
        su *= inv_d;
        sx *= inv_d;
        for (int at = 0; at < d; at += PANEL) {
            take(at);
#pragma unroll
            for (int k = 0; k < NE; ++k) g[k] = rstd * fmaf(-xh[k], sx, g[k] * w[k] - su);
            store_columns<S>(dx + at, d - at, lane, g);
        }
    }
    if (!a.partial || !first) return;
#pragma unroll
    for (int k = 0; k < NE; ++k) g[k] = 0.f;
    for (int at = 0; at < d; at += PANEL) {
        store_columns<S>(pw + at, d - at, lane, g);
        store_columns<S>(pb + at, d - at, lane, g);
    }
}

// Sums of the workgroups' partial sums, in 64 bits: 32 columns a workgroup (whole cache lines; with 8, 500 parts of 6000 columns take
// 10.5 instead of 6.3 us), each by 32 threads that take every 32nd part; added up over the wave, then over the workgroup's waves in
// order.
__global__ void __launch_bounds__(1024) k_norm_sums(NormParams a) {
    constexpr int C = 32, SLICES = 1024 / C;
    __shared__ double box[16][C];
    const int col = threadIdx.x % C, slice = threadIdx.x / C;
    const int64_t c = (int64_t)blockIdx.x * C + col;
    const int64_t width = 2 * (int64_t)a.dim;
    double s = 0.0;
    if (c < width) {
#pragma unroll 8
        for (int p = slice; p < a.parts; p += SLICES) s += (double)a.partial[p * width + c];
    }
#pragma unroll
    for (int k = C; k < kWave; k <<= 1) s += __shfl_xor(s, k, kWave);
    if (lane_id() < C) box[threadIdx.x / kWave][col] = s;
    __syncthreads();
    if (slice || c >= width) return;
    s = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += box[k][col];
    put_sum(a, c, s);
}

// Workgroups of the backward pass.  With sums wanted, each writes 8 bytes a column, which the second kernel reads again: two a
// compute unit (one of the long rows' large workgroups) keep enough loads in flight, and their sums stay a small share of what the
// rows take.  (Twice as many: 16384 x 4096 bf16 96 against 82 us, 4096 x 16384 124 against 111.)
//
// Where one workgroup is done in kAloneTurns turns, it is alone and writes the gradients itself, which saves a launch.  (64 x 400, four
// turns: 7.3 against 8.7 us; two: 5.4 against 8.4; eight: 11.7 against 8.6)
constexpr int kAloneTurns = 4;
int norm_parts(int64_t rows, int32_t dim) {
    int64_t need = rows, most = 256;
    if (dim <= kNormRowMax)
        for_shape<2, 512>(dim, [&](auto s) {
            typedef decltype(s) S;
            need = (rows + S::groups * S::R - 1) / (S::groups * S::R);
            if (S::T <= 256) most = 512;
            if (S::groups > 1 && need <= kAloneTurns) most = 1;
            return 0;
        });
    return (int)(need < most ? need : most);
}
// (shapes of several rows a workgroup add those up in LDS on the way)
static bool sums_alone(int64_t rows, int32_t dim) { return dim <= 1024 && norm_parts(rows, dim) == 1; }

hipError_t launch_norm_backward(hipStream_t st, const NormParams& a) {
    if (a.rows > 0 && a.status && a.dim > kTableRowMax) return hipErrorInvalidValue;
    if (a.rows > 0) {
        hipError_t e = for_types(a.x_type, a.dy_type, [&](auto xt, auto yt) {
            typedef decltype(xt) XT;
            typedef decltype(yt) YT;
            if (a.dim > kNormRowMax) {
                if (a.dim % 4 == 0) k_norm_backward_long<XT, YT, QUADS><<<norm_parts(a.rows, a.dim), 1024, 0, st>>>(a);
                else k_norm_backward_long<XT, YT, RAGGED><<<norm_parts(a.rows, a.dim), 1024, 0, st>>>(a);
            } else {
                for_shape<2, 512>(a.dim, [&](auto s) {
                    typedef decltype(s) S;
                    const int64_t need = (a.rows + S::groups * S::R - 1) / (S::groups * S::R), most = 256 * 2048 / S::threads;
                    const unsigned grid = a.partial ? (unsigned)a.parts : (unsigned)(need < most ? need : most);
                    if (!a.status) k_norm_backward<XT, YT, S, false><<<grid, S::threads, 0, st>>>(a);
                    else if constexpr (std::is_same<XT, float>::value && S::LOW < kTableRowMax) k_norm_backward<XT, YT, S, true><<<grid, S::threads, 0, st>>>(a);
                    return 0;
                });
            }
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    if ((!a.dweight && !a.dbias) || (a.rows > 0 && sums_alone(a.rows, a.dim))) return hipSuccess;
    k_norm_sums<<<(unsigned)((2 * (int64_t)a.dim + 31) / 32), 1024, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace legend
