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

__global__ void __launch_bounds__(256) k_grad_squares(AdamParams a) {
    __shared__ double box[4];
    double s = 0.0;
    for (int64_t u = blockIdx.x; u < a.units; u += gridDim.x) {
        const AdamTensor& t = a.tensors[a.unit_tensor[u]];
        const void* grad = a.grads[t.index];
        const int64_t lo = (u - t.first_unit) * a.unit_elems;
        const int64_t hi = lo + a.unit_elems < t.count ? lo + a.unit_elems : t.count;
        for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
            const double g = (double)load_as(grad, i, t.grad_type);
            s += g * g;
        }
    }
    s = block_sum(s, box);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(256) k_adamw(AdamParams a, int norm_parts) {
    __shared__ double box[4];
    // the state before this step; the last workgroup to be done writes the next one over it
    const double inv_bias1 = a.state->inv_bias1;
    const float inv_bias2_root = a.state->inv_bias2_root;
    const uint64_t key = a.state->key;
    float scale = a.grad_scale ? *a.grad_scale : 1.f;
    bool skip = false;
    if (a.with_norm) {
        double s = 0.0;
        for (int k = threadIdx.x; k < norm_parts; k += 256) s += a.partial[k];
        const double norm = sqrt(block_sum(s, box)) * fabs((double)scale);
        skip = !(fabs(norm) < __builtin_inf());
        if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
        if (a.max_norm > 0.0 && norm > a.max_norm) scale = (float)(a.max_norm / (norm + 1e-6)) * scale;
    }
    const double lr = a.lr * (a.lr_factor ? (double)*a.lr_factor : 1.0);
    const float b1 = (float)a.beta1, b2 = (float)a.beta2, c1 = (float)(1.0 - a.beta1), c2 = (float)(1.0 - a.beta2);
    const float eps = (float)a.eps;
    const int lane = lane_id(), wave = threadIdx.x / kWave;

    for (int64_t u = skip ? a.units : blockIdx.x; u < a.units; u += gridDim.x) {
        const AdamTensor t = a.tensors[a.unit_tensor[u]];
        const void* grad = a.grads[t.index];
        const double tlr = lr * t.lr_scale;
        const float rate = (float)(tlr * inv_bias1), keep = (float)(1.0 - tlr * t.weight_decay);
        const int64_t unit_lo = (u - t.first_unit) * a.unit_elems;
        const int64_t unit_hi = unit_lo + a.unit_elems < t.count ? unit_lo + a.unit_elems : t.count;
        const uint64_t tensor_key = hash_fold(key, (uint64_t)t.index);
        for (int64_t lo = unit_lo + wave * kAdamBlock; lo < unit_hi; lo += 4 * kAdamBlock) {
            const bool block = t.state_type == LEGEND_STATE_BLOCK;
            float m[4], root[4], top_m = 0.f, top_root = 0.f;
            const float old_ms = block ? t.m_scale[lo / kAdamBlock] : 1.f, old_vs = block ? t.v_scale[lo / kAdamBlock] : 1.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t i = lo + j * kWave + lane;
                m[j] = root[j] = 0.f;
                if (i >= unit_hi) continue;
                const float g = load_as(grad, i, t.grad_type) * scale;
                float v;
                if (block) {
                    m[j] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.m)[i], 0) * old_ms;
                    const float r = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.v)[i], 0) * old_vs;
                    v = r * r;
                } else {
                    m[j] = static_cast<const float*>(t.m)[i];
                    v = static_cast<const float*>(t.v)[i];
                }
                m[j] = b1 * m[j] + c1 * g;
                v = b2 * v + (c2 * g) * g;
                root[j] = sqrtf(v);
                float p = t.master ? t.master[i] : load_as(t.param, i, t.param_type);
                p = p * keep - rate * (m[j] / (root[j] * inv_bias2_root + eps));
                if (t.master) t.master[i] = p;
                store_as(t.param, i, t.param_type, p);
                if (!block) {
                    static_cast<float*>(t.m)[i] = m[j];
                    static_cast<float*>(t.v)[i] = v;
                }
                if (fabsf(m[j]) < __builtin_inff()) top_m = fmaxf(top_m, fabsf(m[j]));
                if (root[j] < __builtin_inff()) top_root = fmaxf(top_root, root[j]);
            }
            if (!block) continue;
            float ms = wave_max(top_m) / kTopCode, vs = wave_max(top_root) / kTopCode;
            ms = ms > kLeastScale ? ms : 0.f;
            vs = vs > kLeastScale ? vs : 0.f;
            const float inv_m = ms > 0.f ? 1.f / ms : 0.f, inv_v = vs > 0.f ? 1.f / vs : 0.f;
            const uint32_t block_key = (uint32_t)tensor_key ^ (uint32_t)(lo >> 32) * 0x9E3779B1u;   // a block never crosses 2^32
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t i = lo + j * kWave + lane;
                if (i >= unit_hi) continue;
                const uint32_t w = random_word((uint32_t)i ^ block_key);
                static_cast<uint8_t*>(t.m)[i] = to_code(m[j] * inv_m, fabsf(m[j]) < __builtin_inff(), w);
                const float x = root[j] * inv_v;
                static_cast<uint8_t*>(t.v)[i] = to_code(x > 0.f ? fmaxf(x, kLeastCode) : x, root[j] < __builtin_inff(), w << 16);
            }
            if (lane == 0) {
                t.m_scale[lo / kAdamBlock] = ms;
                t.v_scale[lo / kAdamBlock] = vs;
            }
        }
    }

    // Every workgroup has read the state before it counts itself; no memory needs to be ordered for the last one.
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t done = __hip_atomic_fetch_add(&a.state->ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (done + 1 == gridDim.x) {
            a.state->ticket = 0;
            if (skip) {
                a.state->skipped += 1;
            } else {
                const int64_t steps = a.state->steps + 1;
                a.state->steps = steps;
                a.state->inv_bias1 = 1.0 / (1.0 - pow(a.beta1, (double)(steps + 1)));
                a.state->inv_bias2_root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)(steps + 1))));
                a.state->key = hash_fold(a.seed, (uint64_t)(steps + 1));
            }
        }
    }
}

int adam_unit_elems(int64_t total) {
    (void)total;
    return 4 * kAdamBlock;
}

void adam_state_at(AdamState* s, int64_t steps, double beta1, double beta2, uint64_t seed) {
    *s = AdamState{};
    s->steps = steps;
    s->inv_bias1 = 1.0 / (1.0 - std::pow(beta1, (double)(steps + 1)));
    s->inv_bias2_root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)(steps + 1))));
    s->key = hash_fold(seed, (uint64_t)(steps + 1));
}

hipError_t launch_adamw(hipStream_t st, const AdamParams& a) {
    const int parts = (int)(a.units < kAdamNormParts ? a.units : kAdamNormParts);
    if (a.with_norm && parts > 0) {
        k_grad_squares<<<parts, 256, 0, st>>>(a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t grid = a.units < 1 ? 1 : (a.units < 2048 ? a.units : 2048);
    k_adamw<<<(unsigned)grid, 256, 0, st>>>(a, parts);
    return hipGetLastError();
}

}  // namespace legend
