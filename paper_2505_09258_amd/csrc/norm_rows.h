// What the layer norm kernels share: where a row lies, how its columns are dealt to threads, sums over the threads of a row.
#pragma once

#include "legend_internal.h"
#include "device_utils.h"
#include "tensor_types.h"

namespace legend {

constexpr float kLeftShare = 9.765625e-4f;   // 2^-10: the difference then loses a thousandth of a bit

// A row of a table by its id, or null (and its bit in *status) for one that the call may not read.
__device__ inline const float* table_row(const NormParams& a, int64_t id, bool reports) {
    if (id < 0 || id >= a.table_rows) {
        if (reports) atomicOr(a.status, 1u);
        return nullptr;
    }
    if (a.rel_base) return a.rel_base + id * a.dim;
    // (a 64-bit division takes ten times the instructions of a 32-bit one)
    const int64_t p = a.table_rows <= 0xffffffffll ? (int64_t)((uint32_t)id / (uint32_t)a.rows_per_partition) : id / a.rows_per_partition;
    const float* base = a.part_base[p];
    if (!base) {
        if (reports) atomicOr(a.status, 2u);
        return nullptr;
    }
    return base + (id - p * a.rows_per_partition) * a.dim;
}

// The rows of a call, R at a time, as the kernels ask for them: of a table, the ids a turn ahead of the rows that they name.
template <class XT, bool TABLE, int R>
struct RowSource {
    int64_t id[R];
    __device__ void name(const NormParams& a, int64_t r0) {
        if (!TABLE) return;
#pragma unroll
        for (int i = 0; i < R; ++i) id[i] = a.ids && r0 + i < a.rows ? a.ids[r0 + i] : r0 + i;
    }
    // row r0 + i of the named ones; null behind the last row too
    __device__ const XT* row(const NormParams& a, int64_t r0, int i, bool reports) const {
        if (r0 + i >= a.rows) return nullptr;
        if (!TABLE) return static_cast<const XT*>(a.x) + (r0 + i) * a.x_stride;
        return reinterpret_cast<const XT*>(table_row(a, id[i], reports));
    }
};

template <int CTRL>
__device__ inline float dpp_move(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

// Sum over T neighbouring lanes (8, 16, 32 or 64), in all of them: within a row of 16 lanes by data-parallel moves, across
// rows by swaps of lane groups; no LDS.
template <int T>
__device__ inline float lanes_sum(float v) {
    v += dpp_move<0xB1>(v);                  // lane ^ 1
    v += dpp_move<0x4E>(v);                  // lane ^ 2
    v += dpp_move<0x141>(v);                 // mirrored within 8
    if (T >= 16) v += dpp_move<0x140>(v);    // mirrored within 16
    if (T >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if (T >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// Sum of one number, or sums of two, over the T threads of a row, in all of them.  Rows of more than a wave have the workgroup to
// themselves; `turn` alternates between two boxes, so that one barrier a sum is enough.
template <int T, int N>
__device__ inline void row_sum(float& p, float& q, float (*box)[32], int& turn) {
    p = lanes_sum<(T < kWave ? T : kWave)>(p);
    if (N > 1) q = lanes_sum<(T < kWave ? T : kWave)>(q);
    if (T <= kWave) return;
    constexpr int W = T / kWave;
    float* b = box[turn];
    turn ^= 1;
    if (lane_id() == 0) {
        b[threadIdx.x / kWave] = p;
        if (N > 1) b[16 + threadIdx.x / kWave] = q;
    }
    __syncthreads();
    p = b[0];
#pragma unroll
    for (int k = 1; k < W; ++k) p += b[k];
    if (N < 2) return;
    q = b[16];
#pragma unroll
    for (int k = 1; k < W; ++k) q += b[16 + k];
}

// How a row is dealt to threads: NE columns a thread, T threads a row, R rows at a time, rows of more than LOW columns, WG threads a
// workgroup at least.  Columns go in groups of four, one 16- or 8-byte access at whatever address.  QUADS: dimensions that are a
// multiple of four; accesses behind the row's end go to its last four columns instead and count for nothing.  RAGGED: the others;
// the group that holds the row's end reads the row's last four columns too, and only those count that are no other group's.
// SINGLE: fewer than four columns, one by one.
enum NormColumns { QUADS, RAGGED, SINGLE };
template <int NE_, int T_, int R_, int LOW_, NormColumns MODE_, int WG_>
struct NormShape {
    static constexpr int NE = NE_, T = T_, R = R_, LOW = LOW_;
    static constexpr NormColumns MODE = MODE_;
    static constexpr int threads = T_ < WG_ ? WG_ : T_;      // of a workgroup
    static constexpr int groups = threads / T_;              // rows that a workgroup holds at a time, R times over
    // the group of four that number k of a thread belongs to: the first column that is its own, and the first that it reads
    static __device__ int own(int k, int lane) { return MODE == SINGLE ? k * T + lane : (k >> 2) * (4 * T) + lane * 4; }
    static __device__ int first(int k, int lane, int dim) {
        const int c = own(k, lane), last = MODE == SINGLE ? dim - 1 : dim - 4;
        return always(k) || c < last ? c : last;
    }
    static __device__ int column(int k, int lane, int dim) { return first(k, lane, dim) + (MODE == SINGLE ? 0 : k & 3); }
    // every thread's number k lies in the row, whatever its dimension
    static constexpr __device__ bool always(int k) { return MODE == SINGLE ? (k + 1) * T <= LOW : ((k >> 2) + 1) * (4 * T) <= LOW; }
    static __device__ bool inside(int k, int lane, int dim) {
        if (always(k)) return true;
        if (MODE == RAGGED) return (k & 3) >= own(k, lane) - (dim - 4) || own(k, lane) <= dim - 4;
        return own(k, lane) < dim;
    }
};
constexpr int kTableRowMax = 512;            // columns of a table's rows at most
constexpr int kNormRowMax = 16384;           // longer rows do not fit a workgroup's registers

// Threads and columns a thread for every dimension: a wave and less while a row fits its registers with room for the next one's, then
// workgroups of 256 and 512 (1024 hold fewer of each other's loads in flight: 8192 x 8192 bf16 75 against 52 us forward, 100 against 83
// backward).  R: rows of at most 512 columns that a thread group takes at a time (forward 1, 50 000 x 100 table rows 11.8 us against 15.4
// with 4; backward 2, 500 000 x 100 111 against 135 with 1); WG: threads of a workgroup where a row needs no more than a wave
template <int R, int WG, NormColumns Q, class F>
auto for_columns(int dim, F&& f) {
    if (dim <= 32) return f(NormShape<4, 8, R, 0, Q, WG>{});
    if (dim <= 64) return f(NormShape<4, 16, R, 32, Q, WG>{});
    if (dim <= 128) return f(NormShape<4, 32, R, 64, Q, WG>{});
    if (dim <= 256) return f(NormShape<4, 64, R, 128, Q, WG>{});
    if (dim <= 512) return f(NormShape<8, 64, R, 256, Q, WG>{});
    if (dim <= 1024) return f(NormShape<16, 64, 1, 512, Q, WG>{});
    if (dim <= 2048) return f(NormShape<8, 256, 1, 1024, Q, 256>{});
    if (dim <= 4096) return f(NormShape<16, 256, 1, 2048, Q, 256>{});
    if (dim <= 8192) return f(NormShape<16, 512, 1, 4096, Q, 512>{});
    return f(NormShape<32, 512, 1, 8192, Q, 512>{});
}
template <int R, int WG, class F>
auto for_shape(int dim, F&& f) {
    if (dim < 4) return f(NormShape<4, 8, R, 0, SINGLE, WG>{});
    return dim % 4 == 0 ? for_columns<R, WG, QUADS>(dim, f) : for_columns<R, WG, RAGGED>(dim, f);
}

// A thread's columns of a row as they lie in memory; no branch between the loads.  `inside` says which numbers count.
template <class E, class S>
struct RowColumns {
    typedef E quad __attribute__((ext_vector_type(4)));
    quad v[S::NE / 4];
    __device__ void load(const E* row, int dim, int lane) {
        if (S::MODE != SINGLE) {
#pragma unroll
            for (int k = 0; k < S::NE; k += 4) v[k / 4] = *reinterpret_cast<const typename Quad<E>::type*>(row + S::first(k, lane, dim));
        } else {
#pragma unroll
            for (int k = 0; k < S::NE; ++k) v[k / 4][k % 4] = row[S::first(k, lane, dim)];
        }
    }
    __device__ void clear() {
#pragma unroll
        for (int k = 0; k < S::NE / 4; ++k) v[k] = (quad)(E)0.f;
    }
    __device__ float number(int k) const { return (float)v[k / 4][k % 4]; }
};

template <class S, class E>
__device__ inline void store_columns(E* row, int dim, int lane, const float* in) {
    if (S::MODE != SINGLE) {
#pragma unroll
        for (int k = 0; k < S::NE; k += 4) {
            const int c = S::own(k, lane);
            if (S::always(k) || c <= dim - 4) {
                store_quad(row + c, in + k);
            } else if (S::MODE == RAGGED && c < dim) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (S::inside(k + j, lane, dim)) row[S::column(k + j, lane, dim)] = (E)in[k + j];
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < S::NE; ++k)
            if (S::inside(k, lane, dim)) row[S::column(k, lane, dim)] = (E)in[k];
    }
}

// weight or bias as fp32, from column `at` on, `none` where there is none
template <class S>
__device__ inline void load_parameter(const void* p, int type, float none, int dim, int lane, float* out, int at = 0) {
    auto take = [&](auto e) {
        RowColumns<decltype(e), S> r;
        r.load(static_cast<const decltype(e)*>(p) + at, dim, lane);
#pragma unroll
        for (int k = 0; k < S::NE; ++k) out[k] = r.number(k);
    };
    if (!p) {
#pragma unroll
        for (int k = 0; k < S::NE; ++k) out[k] = none;
    } else if (type == LEGEND_TYPE_FLOAT) {
        take(float{});
    } else if (type == LEGEND_TYPE_BFLOAT) {
        take(bf16_t{});
    } else {
        take(half_t{});
    }
}

template <class F>
hipError_t for_types(int x_type, int y_type, F&& f) {
    if (x_type == LEGEND_TYPE_FLOAT) {
        if (y_type == LEGEND_TYPE_FLOAT) return f(float{}, float{});
        if (y_type == LEGEND_TYPE_BFLOAT) return f(float{}, bf16_t{});
        return f(float{}, half_t{});
    }
    if (x_type == LEGEND_TYPE_BFLOAT) return y_type == LEGEND_TYPE_FLOAT ? f(bf16_t{}, float{}) : f(bf16_t{}, bf16_t{});
    return y_type == LEGEND_TYPE_FLOAT ? f(half_t{}, float{}) : f(half_t{}, half_t{});
}

}  // namespace legend
