// AdamW over many tensors in one launch, with the norm of all gradients in a launch before it where it is asked for.
//
// Every tensor is cut into units of unit_elems elements, the last one partial; a workgroup takes units in turn, so that
// hundreds of small tensors and a few large ones fill the card alike.  Nothing is exchanged between workgroups: each adds up the
// partial sums of the norm by itself (8 KB from L2), in one order, in 64 bits.
//
// 8-bit states: a wave owns a block of 256 elements; its largest |m| and sqrt(v) set the block's scales.
#include "legend_internal.h"
#include "device_utils.h"
#include "tensor_types.h"

#include <cmath>

namespace legend {

constexpr float kTopCode = 448.f;           // largest e4m3 value
constexpr float kLeastCode = 0.001953125f;  // smallest above zero, 2^-9
constexpr float kLeastScale = 7.8886091e-31f;  // 2^-100: 1 / scale stays far from infinity

constexpr int64_t kLargeTotal = 4 << 20;    // elements
constexpr int64_t kStepGrid = 2048;         // workgroups of a step: eight a compute unit

__device__ inline float wave_max(float v) {
#pragma unroll
    for (int k = 1; k < kWave; k <<= 1) v = fmaxf(v, wave_shfl_xor(v, k));
    return v;
}

// sum of 256 threads' doubles, in every thread
__device__ inline double block_sum(double v, double* box) {
#pragma unroll
    for (int k = 1; k < kWave; k <<= 1) v += __shfl_xor(v, k, kWave);
    if (lane_id() == 0) box[threadIdx.x / kWave] = v;
    __syncthreads();
    v = (box[0] + box[1]) + (box[2] + box[3]);
    __syncthreads();
    return v;
}

__device__ inline uint32_t random_word(uint32_t w) {
    w ^= w >> 16;
    w *= 0x9E3779B1u;
    w ^= w >> 15;
    w *= 0x85157AF5u;
    return w ^ (w >> 16);
}

// e4m3 code of x in units of its scale; the conversion adds the word's upper 20 bits below the last bit that it keeps
__device__ inline uint8_t to_code(float x, bool finite, uint32_t word) {
    x = finite ? fminf(fmaxf(x, -kTopCode), kTopCode) : __builtin_nanf("");
    return (uint8_t)__builtin_amdgcn_cvt_sr_fp8_f32(x, word, 0, 0);
}

// What a step has in common for all elements of a tensor.
struct Step {
    float scale, b1, b2, c1, c2, eps, inv_bias2_root;    // of the gradient; beta and 1 - beta; epsilon
    float rate, keep;                                    // lr' / (1 - beta1^t), 1 - lr' weight_decay
    uint32_t key;
};

// The tables are constant while a kernel runs and their indices are the same for a whole workgroup: scalar loads.
typedef const __attribute__((address_space(4))) AdamTensor* TensorTable;
typedef const __attribute__((address_space(4))) int32_t* UnitTable;
typedef const void* const __attribute__((address_space(4)))* GradTable;

__device__ inline AdamTensor tensor_at(TensorTable p) {
    return AdamTensor{p->param, p->master, p->m, p->v, p->m_scale, p->v_scale, p->count, p->first_unit, p->weight_decay, p->lr_scale,
                      p->param_type, p->grad_type, p->state_type, p->index};
}

// Four consecutive elements as they lie in memory, and as numbers.
__device__ inline uint4 raw_quad(const void* p, int64_t i, int type) {
    typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t four __attribute__((ext_vector_type(4), aligned(4)));
    if (type == LEGEND_TYPE_FLOAT) {
        const four v = *reinterpret_cast<const four*>(static_cast<const float*>(p) + i);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    const two v = *reinterpret_cast<const two*>(static_cast<const uint16_t*>(p) + i);
    return make_uint4(v.x, v.y, 0u, 0u);
}
__device__ inline void numbers_of(uint4 r, int type, float* out) {
    if (type == LEGEND_TYPE_FLOAT) {
        out[0] = __uint_as_float(r.x); out[1] = __uint_as_float(r.y); out[2] = __uint_as_float(r.z); out[3] = __uint_as_float(r.w);
    } else if (type == LEGEND_TYPE_BFLOAT) {
        out[0] = __uint_as_float(r.x << 16); out[1] = __uint_as_float(r.x & 0xffff0000u);
        out[2] = __uint_as_float(r.y << 16); out[3] = __uint_as_float(r.y & 0xffff0000u);
    } else {
        typedef half_t h2 __attribute__((ext_vector_type(2)));
        const h2 lo = __builtin_bit_cast(h2, r.x), hi = __builtin_bit_cast(h2, r.y);
        out[0] = (float)lo.x; out[1] = (float)lo.y; out[2] = (float)hi.x; out[3] = (float)hi.y;
    }
}
__device__ inline void put_quad(void* p, int64_t i, int type, const float* v) {
    if (type == LEGEND_TYPE_FLOAT) store_quad(static_cast<float*>(p) + i, v);
    else if (type == LEGEND_TYPE_BFLOAT) store_quad(static_cast<bf16_t*>(p) + i, v);
    else store_quad(static_cast<half_t*>(p) + i, v);
}

// Moments and parameter of one element; the root of the new second moment comes back.
__device__ inline float step_element(const Step& s, float g, float& m, float& v, float& p) {
    g *= s.scale;
    m = s.b1 * m + s.c1 * g;
    v = s.b2 * v + (s.c2 * g) * g;
    const float root = sqrtf(v);
    p = p * s.keep - s.rate * (m / (root * s.inv_bias2_root + s.eps));
    return root;
}

// Scale of a block from its lanes' largest finite magnitudes, and its reciprocal.
__device__ inline float block_scale(float top, float& inverse) {
    float s = wave_max(top) / kTopCode;
    s = s > kLeastScale ? s : 0.f;
    inverse = s > 0.f ? 1.f / s : 0.f;
    return s;
}
__device__ inline float finite_or_zero(float v) { return v < __builtin_inff() ? v : 0.f; }
__device__ inline void codes_of(float m, float inv_m, float root, float inv_root, uint32_t word, uint8_t& cm, uint8_t& cr) {
    cm = to_code(m * inv_m, fabsf(m) < __builtin_inff(), word);
    const float x = root * inv_root;
    cr = to_code(x > 0.f ? fmaxf(x, kLeastCode) : x, root < __builtin_inff(), word << 16);
}
__device__ inline uint32_t block_key(const Step& s, int64_t lo) { return s.key ^ (uint32_t)(lo >> 32) * 0x9E3779B1u; }   // a block never crosses 2^32

// K whole blocks of 256 elements, `apart` elements from one to the next: every load first, then the arithmetic.
template <int K, bool BLOCK>
__device__ inline void whole_blocks(const AdamTensor& t, const void* grad, const Step& s, int64_t lo, int64_t apart) {
    const int64_t i0 = lo + lane_id() * 4;
    const int ptype = t.master ? (int)LEGEND_TYPE_FLOAT : t.param_type;
    const void* from = t.master ? t.master : t.param;
    uint4 rg[K], rp[K], rm[K], rv[K];
    uint32_t cm[K], cv[K];
    float ms[K], vs[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t i = i0 + k * apart;
        rg[k] = raw_quad(grad, i, t.grad_type);
        rp[k] = raw_quad(from, i, ptype);
        if (BLOCK) {
            typedef uint32_t word __attribute__((aligned(1)));
            cm[k] = *reinterpret_cast<const word*>(static_cast<const uint8_t*>(t.m) + i);
            cv[k] = *reinterpret_cast<const word*>(static_cast<const uint8_t*>(t.v) + i);
            ms[k] = t.m_scale[(lo + k * apart) / kAdamBlock];
            vs[k] = t.v_scale[(lo + k * apart) / kAdamBlock];
        } else {
            rm[k] = raw_quad(t.m, i, LEGEND_TYPE_FLOAT);
            rv[k] = raw_quad(t.v, i, LEGEND_TYPE_FLOAT);
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t i = i0 + k * apart;
        float g[4], p[4], m[4], v[4], root[4];
        numbers_of(rg[k], t.grad_type, g);
        numbers_of(rp[k], ptype, p);
        if (BLOCK) {
            m[0] = __builtin_amdgcn_cvt_f32_fp8(cm[k], 0) * ms[k]; m[1] = __builtin_amdgcn_cvt_f32_fp8(cm[k], 1) * ms[k];
            m[2] = __builtin_amdgcn_cvt_f32_fp8(cm[k], 2) * ms[k]; m[3] = __builtin_amdgcn_cvt_f32_fp8(cm[k], 3) * ms[k];
            v[0] = __builtin_amdgcn_cvt_f32_fp8(cv[k], 0) * vs[k]; v[1] = __builtin_amdgcn_cvt_f32_fp8(cv[k], 1) * vs[k];
            v[2] = __builtin_amdgcn_cvt_f32_fp8(cv[k], 2) * vs[k]; v[3] = __builtin_amdgcn_cvt_f32_fp8(cv[k], 3) * vs[k];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= v[j];
        } else {
            numbers_of(rm[k], LEGEND_TYPE_FLOAT, m);
            numbers_of(rv[k], LEGEND_TYPE_FLOAT, v);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) root[j] = step_element(s, g[j], m[j], v[j], p[j]);
        if (t.master) store_quad(t.master + i, p);
        put_quad(t.param, i, t.param_type, p);
        if (!BLOCK) {
            store_quad(static_cast<float*>(t.m) + i, m);
            store_quad(static_cast<float*>(t.v) + i, v);
            continue;
        }
        float top_m = 0.f, top_root = 0.f, inv_m, inv_root;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            top_m = fmaxf(top_m, finite_or_zero(fabsf(m[j])));
            top_root = fmaxf(top_root, finite_or_zero(root[j]));
        }
        const float new_ms = block_scale(top_m, inv_m), new_vs = block_scale(top_root, inv_root);
        const uint32_t key = block_key(s, lo + k * apart);
        uint32_t wm = 0, wr = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint8_t a, b;
            codes_of(m[j], inv_m, root[j], inv_root, random_word((uint32_t)(i + j) ^ key), a, b);
            wm |= (uint32_t)a << (8 * j);
            wr |= (uint32_t)b << (8 * j);
        }
        typedef uint32_t word __attribute__((aligned(1)));
        *reinterpret_cast<word*>(static_cast<uint8_t*>(t.m) + i) = wm;
        *reinterpret_cast<word*>(static_cast<uint8_t*>(t.v) + i) = wr;
        if (lane_id() == 0) {
            t.m_scale[(lo + k * apart) / kAdamBlock] = new_ms;
            t.v_scale[(lo + k * apart) / kAdamBlock] = new_vs;
        }
    }
}

// The last block of a tensor, elements [lo, count): single elements, neighbours in neighbouring lanes.
__device__ inline void part_block(const AdamTensor& t, const void* grad, const Step& s, int64_t lo) {
    const bool block = t.state_type == LEGEND_STATE_BLOCK;
    const float ms = block ? t.m_scale[lo / kAdamBlock] : 1.f, vs = block ? t.v_scale[lo / kAdamBlock] : 1.f;
    float m[4], root[4], top_m = 0.f, top_root = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = lo + j * kWave + lane_id();
        m[j] = root[j] = 0.f;
        if (i >= t.count) continue;
        float v;
        if (block) {
            m[j] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.m)[i], 0) * ms;
            v = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.v)[i], 0) * vs;
            v *= v;
        } else {
            m[j] = static_cast<const float*>(t.m)[i];
            v = static_cast<const float*>(t.v)[i];
        }
        float p = t.master ? t.master[i] : load_as(t.param, i, t.param_type);
        root[j] = step_element(s, load_as(grad, i, t.grad_type), m[j], v, p);
        if (t.master) t.master[i] = p;
        store_as(t.param, i, t.param_type, p);
        if (!block) {
            static_cast<float*>(t.m)[i] = m[j];
            static_cast<float*>(t.v)[i] = v;
        }
        top_m = fmaxf(top_m, finite_or_zero(fabsf(m[j])));
        top_root = fmaxf(top_root, finite_or_zero(root[j]));
    }
    if (!block) return;
    float inv_m, inv_root;
    const float new_ms = block_scale(top_m, inv_m), new_vs = block_scale(top_root, inv_root);
    const uint32_t key = block_key(s, lo);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = lo + j * kWave + lane_id();
        if (i < t.count)
            codes_of(m[j], inv_m, root[j], inv_root, random_word((uint32_t)i ^ key), static_cast<uint8_t*>(t.m)[i], static_cast<uint8_t*>(t.v)[i]);
    }
    if (lane_id() == 0) {
        t.m_scale[lo / kAdamBlock] = new_ms;
        t.v_scale[lo / kAdamBlock] = new_vs;
    }
}

// What a step reads of the state and what it leaves lie apart: its first kernel (this one's first thread, in the kernel of the
// squares, or alone) makes the one from the other, its last writes the other.  No workgroup waits for another, and a counter of
// finished workgroups, which would tell the last one, costs 10 ns for each of them.
__device__ inline void begin_step(const AdamParams& a) {
    AdamState& st = *a.state;
    st.inv_bias1 = 1.0 / (1.0 - st.power1);
    st.inv_bias2_root = (float)(1.0 / sqrt(1.0 - st.power2));
    st.key = hash_fold(a.seed, (uint64_t)(st.steps + 1));
    st.now_steps = st.steps;
    st.now_skipped = st.skipped;
    st.now_power1 = st.power1;
    st.now_power2 = st.power2;
}
__global__ void k_begin_step(AdamParams a) { begin_step(a); }

// K: blocks that a wave takes of a unit (unit_elems = 4 K blocks).
template <int K>
__global__ void __launch_bounds__(256) k_grad_squares(AdamParams a) {
    __shared__ double box[4];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (blockIdx.x == 0 && threadIdx.x == 0) begin_step(a);
    const TensorTable tensors = (TensorTable)a.tensors;
    const UnitTable units = (UnitTable)a.unit_tensor;
    const GradTable grads = (GradTable)a.grads;
    for (int64_t u = blockIdx.x; u < a.units; u += gridDim.x) {
        const int k0 = units[u];
        const int64_t count = tensors[k0].count, lo = (u - tensors[k0].first_unit) * (K * 1024);
        const int type = tensors[k0].grad_type;
        const void* grad = grads[k0];
        if (lo + K * 1024 <= count) {
            uint4 r[K];
#pragma unroll
            for (int k = 0; k < K; ++k) r[k] = raw_quad(grad, lo + k * 1024 + threadIdx.x * 4, type);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float g[4];
                numbers_of(r[k], type, g);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[j] = fma((double)g[j], (double)g[j], s[j]);
            }
        } else {
            for (int64_t i = lo + threadIdx.x; i < count; i += 256) {
                const double g = (double)load_as(grad, i, type);
                s[0] += g * g;
            }
        }
    }
    const double all = block_sum((s[0] + s[1]) + (s[2] + s[3]), box);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = all;
}

template <int K>
__global__ void __launch_bounds__(256) k_adamw(AdamParams a, int norm_parts) {
    __shared__ double box[4];
    const double inv_bias1 = a.state->inv_bias1;
    const uint64_t key = a.state->key;
    Step s;
    s.inv_bias2_root = a.state->inv_bias2_root;
    s.scale = a.grad_scale ? *a.grad_scale : 1.f;
    bool skip = false;
    if (a.with_norm) {
        double sum = 0.0;
        for (int k = threadIdx.x; k < norm_parts; k += 256) sum += a.partial[k];
        const double norm = sqrt(block_sum(sum, box)) * fabs((double)s.scale);
        skip = !(norm < __builtin_inf());
        if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
        if (a.max_norm > 0.0 && norm > a.max_norm) s.scale = (float)(a.max_norm / (norm + 1e-6)) * s.scale;
    }
    const double lr = a.lr * (a.lr_factor ? (double)*a.lr_factor : 1.0);
    s.b1 = (float)a.beta1;
    s.b2 = (float)a.beta2;
    s.c1 = (float)(1.0 - a.beta1);
    s.c2 = (float)(1.0 - a.beta2);
    s.eps = (float)a.eps;
    const int wave = threadIdx.x / kWave;
    const TensorTable tensors = (TensorTable)a.tensors;
    const UnitTable units = (UnitTable)a.unit_tensor;
    const GradTable grads = (GradTable)a.grads;

    for (int64_t u = skip ? a.units : blockIdx.x; u < a.units; u += gridDim.x) {
        const int k0 = units[u];
        const AdamTensor t = tensor_at(tensors + k0);
        const void* grad = grads[k0];
        const double tlr = lr * t.lr_scale;
        s.rate = (float)(tlr * inv_bias1);
        s.keep = (float)(1.0 - tlr * t.weight_decay);
        s.key = (uint32_t)hash_fold(key, (uint64_t)t.index);
        const int64_t unit_lo = (u - t.first_unit) * (K * 1024), lo = unit_lo + wave * kAdamBlock;
        if (unit_lo + K * 1024 <= t.count) {
            if (t.state_type == LEGEND_STATE_BLOCK) whole_blocks<K, true>(t, grad, s, lo, 1024);
            else whole_blocks<K, false>(t, grad, s, lo, 1024);
        } else {
            for (int k = 0; k < K; ++k) {
                const int64_t at = lo + k * 1024;
                if (at >= t.count) break;
                if (at + kAdamBlock > t.count) part_block(t, grad, s, at);
                else if (t.state_type == LEGEND_STATE_BLOCK) whole_blocks<1, true>(t, grad, s, at, 0);
                else whole_blocks<1, false>(t, grad, s, at, 0);
            }
        }
    }

    if (blockIdx.x == 0 && threadIdx.x == 0) {
        AdamState& st = *a.state;
        st.steps = st.now_steps + (skip ? 0 : 1);
        st.skipped = st.now_skipped + (skip ? 1 : 0);
        st.power1 = st.now_power1 * (skip ? 1.0 : a.beta1);
        st.power2 = st.now_power2 * (skip ? 1.0 : a.beta2);
    }
}

// Small sets: units of 1024, so that more workgroups share them.  Large ones: 4096, so that a wave has four blocks' loads in flight.
int adam_unit_elems(int64_t total) { return total >= kLargeTotal ? 4096 : 1024; }

void adam_state_at(AdamState* s, int64_t steps, double beta1, double beta2) {
    *s = AdamState{};
    s->steps = steps;
    s->power1 = std::pow(beta1, (double)(steps + 1));
    s->power2 = std::pow(beta2, (double)(steps + 1));
}

template <int K>
static hipError_t launch_units(hipStream_t st, const AdamParams& a) {
    const int parts = (int)(a.units < kAdamNormParts ? a.units : kAdamNormParts);
    if (a.with_norm && parts > 0) k_grad_squares<K><<<parts, 256, 0, st>>>(a);
    else k_begin_step<<<1, 1, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t grid = a.units < 1 ? 1 : (a.units < kStepGrid ? a.units : kStepGrid);
    k_adamw<K><<<(unsigned)grid, 256, 0, st>>>(a, parts);
    return hipGetLastError();
}

hipError_t launch_adamw(hipStream_t st, const AdamParams& a) {
    return a.unit_elems == 4096 ? launch_units<4>(st, a) : launch_units<1>(st, a);
}

}  // namespace legend
