// What the layer norm kernels share: where a row lies, how its columns are dealt to threads, sums over the threads of a row.
#pragma once

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
    // (a 64-bit division takes ten times the instructions of a 32-bit one)
    const int64_t p = a.table_rows <= 0xffffffffll ? (int64_t)((uint32_t)id / (uint32_t)a.rows_per_partition) : id / a.rows_per_partition;
    const float* base = a.part_base[p];
    if (!base) {
        if (reports) atomicOr(a.status, 2u);
        return nullptr;
    }
    return reinterpret_cast<const XT*>(base + (id - p * a.rows_per_partition) * a.dim);
}

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

// Sums of two numbers over the T threads of a row, in all of them.  Rows of more than a wave have the workgroup to themselves;
// `box` holds 2 x 16 floats, `turn` alternates so that one barrier a sum is enough.
template <int T>
__device__ inline void row_sum2(float& p, float& q, float (*box)[32], int& turn) {
    p = lanes_sum<(T < kWave ? T : kWave)>(p);
    q = lanes_sum<(T < kWave ? T : kWave)>(q);
    if (T <= kWave) return;
    constexpr int W = T / kWave;
    float* b = box[turn];
    turn ^= 1;
    if (lane_id() == 0) {
        b[threadIdx.x / kWave] = p;
        b[16 + threadIdx.x / kWave] = q;
    }
    __syncthreads();
    p = q = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) { p += b[k]; q += b[16 + k]; }
}

// The NE columns of a row that thread `lane` of T holds: groups of four (16- or 8-byte accesses) where the dimension is a
// multiple of four, else single elements, neighbours in neighbouring threads.
template <int NE, int T>
__device__ inline int column_of(int k, int lane, bool quads) { return quads ? (k >> 2) * (4 * T) + lane * 4 + (k & 3) : k * T + lane; }

template <int NE, int T, class E>
__device__ inline void load_columns(const E* row, int dim, int lane, bool quads, float* out) {
    if (quads) {
#pragma unroll
        for (int k = 0; k < NE; k += 4) {
            const int c = column_of<NE, T>(k, lane, true);
            if (c < dim) load_quad(row + c, out + k);
            else out[k] = out[k + 1] = out[k + 2] = out[k + 3] = 0.f;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NE; ++k) {
            const int c = column_of<NE, T>(k, lane, false);
            out[k] = c < dim ? (float)row[c] : 0.f;
        }
    }
}

template <int NE, int T, class E>
__device__ inline void store_columns(E* row, int dim, int lane, bool quads, const float* in) {
    if (quads) {
#pragma unroll
        for (int k = 0; k < NE; k += 4) {
            const int c = column_of<NE, T>(k, lane, true);
            if (c < dim) store_quad(row + c, in + k);
        }
    } else {
#pragma unroll
        for (int k = 0; k < NE; ++k) {
            const int c = column_of<NE, T>(k, lane, false);
            if (c < dim) row[c] = (E)in[k];
        }
    }
}

// weight or bias as fp32, `none` where there is none
template <int NE, int T>
__device__ inline void load_parameter(const void* p, int type, float none, int dim, int lane, bool quads, float* out) {
    if (!p) {
#pragma unroll
        for (int k = 0; k < NE; ++k) out[k] = none;
    } else if (type == LEGEND_TYPE_FLOAT) {
        load_columns<NE, T>(static_cast<const float*>(p), dim, lane, quads, out);
    } else if (type == LEGEND_TYPE_BFLOAT) {
        load_columns<NE, T>(static_cast<const bf16_t*>(p), dim, lane, quads, out);
    } else {
        load_columns<NE, T>(static_cast<const half_t*>(p), dim, lane, quads, out);
    }
}

// How a row of `dim` columns is dealt to threads: f(NE, T, R): NE columns a thread, T threads a row, R rows at a time.
template <int NE_, int T_, int R_>
struct NormShape {
    static constexpr int NE = NE_, T = T_, R = R_;
    static constexpr int threads = T_ < 256 ? 256 : T_;      // of a workgroup
    static constexpr int groups = threads / T_;              // rows that a workgroup holds at a time, R times over
};
constexpr int kNormRowMax = 16384;           // longer rows do not fit a workgroup's registers

template <class F>
auto for_shape(int dim, F&& f) {
    if (dim <= 32) return f(NormShape<4, 8, 4>{});
    if (dim <= 64) return f(NormShape<4, 16, 4>{});
    if (dim <= 128) return f(NormShape<4, 32, 4>{});
    if (dim <= 256) return f(NormShape<4, 64, 4>{});
    if (dim <= 512) return f(NormShape<8, 64, 2>{});
    if (dim <= 1024) return f(NormShape<16, 64, 1>{});
    if (dim <= 2048) return f(NormShape<8, 256, 1>{});
    if (dim <= 4096) return f(NormShape<16, 256, 1>{});
    if (dim <= 8192) return f(NormShape<8, 1024, 1>{});
    return f(NormShape<16, 1024, 1>{});
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
