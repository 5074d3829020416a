// AdamW over many tensors in one launch, with the norm of all gradients in a launch before it where it is asked for.
//
// Every tensor is cut into units of unit_elems elements, the last one partial, so that hundreds of small tensors and a few large
// ones fill the card alike.  The norm's sums are taken in 64 bits and in one order, and no result depends on the order in which
// workgroups run.
//
// 8-bit states: a wave owns a block of 256 elements, four neighbouring ones a lane; its largest |m| and v set the block's scales.
//
// Bound by HBM: 60 M fp32 parameters in 312 us, 5.4 TB/s of what a step cannot do without (first form, one element a thread: 687; with a
// counter of finished workgroups at the end, 10 ns a workgroup: 20 us more); 120 M bf16 parameters with master copies and 8-bit states in
// 345 us, 5.6 TB/s (1476; with divisions and roots as the compiler expands them 490).  The gradients are read twice, the second time from
// the cache where they fit.  Small sets are bound by their launches: 41 000 elements in 8 us, without the norm 5.5.
#include "legend_internal.h"
#include "device_utils.h"
#include "tensor_types.h"

#include <cmath>

namespace legend {

constexpr float kTopCode = 448.f;           // largest e4m3 value
constexpr float kLeastCode = 0.001953125f;  // smallest above zero, 2^-9
constexpr float kLeastScale = 7.8886091e-31f;  // 2^-100: 1 / scale stays far from infinity
constexpr uint32_t kInfinity = 0x7f800000u;  // bits

// Sets of fewer elements are cut into units of 1024, so that more workgroups share them, and their workgroups all fit the card at a
// time; each adds up the norm's partial sums by itself, which is less than a launch takes.  Larger sets are cut into units of 2048, two
// blocks in flight a wave (four: 515 against 417 us for 120 M bf16 parameters with 8-bit states, too many registers; units of 2048 for
// 3 M elements: 28.0 against 24.8), one unit a workgroup while a launch holds them (1024 workgroups that take units in turn: 358 against
// 335 us), and a kernel of one workgroup adds the partial sums up.  adam_grid has the numbers of workgroups.
constexpr int64_t kLargeTotal = 4 << 20;
constexpr int64_t kGridAlone = 256;         // workgroups that count themselves instead of a launch before them
// Workgroups of the kernel of the squares.  (120 M elements: 2048 of them read the gradients at 5 TB/s, 1024 at 3.6; 3 M: 24.7 against
// 25.5 us for the whole step)
constexpr int kPartsSmall = 1024, kPartsLarge = kAdamNormParts;

// Largest of the wave's numbers, of two kinds at a time (data-parallel moves that depend on each other wait), none below zero, in all
// lanes.  Compared as integers, which orders them alike, with infinity and NaN at the top.
template <int CTRL>
__device__ inline void max_moved(uint32_t& a, uint32_t& b) {
    const uint32_t x = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, CTRL, 0xf, 0xf, false);
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, false);
    a = max(a, x);
    b = max(b, y);
}
__device__ inline void wave_max(uint32_t& a, uint32_t& b) {
    max_moved<0xB1>(a, b);                   // lane ^ 1
    max_moved<0x4E>(a, b);                   // lane ^ 2
    max_moved<0x141>(a, b);                  // mirrored within 8
    max_moved<0x140>(a, b);                  // mirrored within 16
    const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const auto q = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    a = max((uint32_t)p[0], (uint32_t)p[1]);
    b = max((uint32_t)q[0], (uint32_t)q[1]);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const auto t = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    a = max((uint32_t)r[0], (uint32_t)r[1]);
    b = max((uint32_t)t[0], (uint32_t)t[1]);
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

// What a step has in common for all elements of a tensor.
struct Step {
    float scale, b1, b2, c1, c2, eps, inv_bias2_root;    // of the gradient; beta and 1 - beta; epsilon
    float rate, keep;                                    // lr' / (1 - beta1^t), 1 - lr' weight_decay
    uint32_t key;
};

__device__ inline void constants_of(const AdamParams& a, Step& s) {
    s.b1 = (float)a.beta1;
    s.b2 = (float)a.beta2;
    s.c1 = (float)(1.0 - a.beta1);
    s.c2 = (float)(1.0 - a.beta2);
    s.eps = (float)a.eps;
}
__device__ inline void rates_of(const AdamTensor& t, double lr, double inv_bias1, uint64_t key, Step& s) {
    const double tlr = lr * t.lr_scale;
    s.rate = (float)(tlr * inv_bias1);
    s.keep = (float)(1.0 - tlr * t.weight_decay);
    s.key = (uint32_t)hash_fold(key, (uint64_t)t.index);
}

// The tables are constant while a kernel runs and their indices are the same for a whole workgroup: scalar loads.
typedef const __attribute__((address_space(4))) AdamTensor* TensorTable;
typedef const __attribute__((address_space(4))) int32_t* UnitTable;
typedef const void* const __attribute__((address_space(4)))* GradTable;

__device__ inline AdamTensor tensor_at(TensorTable p) {
    return AdamTensor{p->param, p->master, p->m, p->v, p->m_scale, p->v_scale, p->count, p->first_unit, p->weight_decay, p->lr_scale,
                      p->param_type, p->grad_type, p->state_type, p->index};
}

// Four consecutive elements as they lie in memory, and as numbers.
template <bool STREAM>
__device__ inline uint4 raw_quad(const void* p, int64_t i, int type) {
    typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t four __attribute__((ext_vector_type(4), aligned(4)));
    if (type == LEGEND_TYPE_FLOAT) {
        const four* q = reinterpret_cast<const four*>(static_cast<const float*>(p) + i);
        const four v = STREAM ? __builtin_nontemporal_load(q) : *q;
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    const two* q = reinterpret_cast<const two*>(static_cast<const uint16_t*>(p) + i);
    const two v = STREAM ? __builtin_nontemporal_load(q) : *q;
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
template <bool STREAM>
__device__ inline void put_quad(void* p, int64_t i, int type, const float* v) {
    if (type == LEGEND_TYPE_FLOAT) store_quad<STREAM>(static_cast<float*>(p) + i, v);
    else if (type == LEGEND_TYPE_BFLOAT) store_quad<STREAM>(static_cast<bf16_t*>(p) + i, v);
    else store_quad<STREAM>(static_cast<half_t*>(p) + i, v);
}
__device__ inline void codes_to_numbers(uint32_t codes, float scale, float* out) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    out[0] = lo[0] * scale; out[1] = lo[1] * scale; out[2] = hi[0] * scale; out[3] = hi[1] * scale;
}

// The step of a parameter from its new moments; the reciprocal is the hardware's, within 1.6 half steps of fp32.
__device__ inline float step_parameter(const Step& s, float m, float root, float p) {
    const float down = m * __builtin_amdgcn_rcpf(fmaf(root, s.inv_bias2_root, s.eps));
    return fmaf(p, s.keep, -(s.rate * down));
}
// 32-bit states: the hardware's root, within 1.6 half steps; a second moment below fp32's normal numbers has the root 0.
__device__ inline void step_float(const Step& s, float g, float& m, float& v, float& p) {
    g *= s.scale;
    m = fmaf(s.b1, m, s.c1 * g);
    v = fmaf(s.b2, v, (s.c2 * g) * g);
    p = step_parameter(s, m, __builtin_amdgcn_sqrtf(v), p);
}

// 8-bit states: every operation up to the code is rounded to nearest once, as it is written (a code depends on the last bit of
// what it is made from: a root or a quotient that is a bit off is another code once in a million).
// Root of v: from the hardware's reciprocal root by one step whose residual is exact; small numbers are lifted, since the residual of one
// below 2^-102 is not.  That this rounds to nearest was compared for all mantissas of both parities of the exponent.  NaN for infinity.
constexpr float kSmallMoment = 0x1p-100f;
__device__ inline float root_step(float v) {
    const float y = __builtin_amdgcn_rsqf(v);
    const float q = v * y;
    return fmaf(fmaf(-q, q, v), 0.5f * y, q);
}
__device__ inline float lifted_root(float v) { return v > 0.f ? root_step(v * 0x1p64f) * 0x1p-32f : v; }
__device__ inline float rounded_root(float v) { return v < kSmallMoment ? lifted_root(v) : root_step(v); }
// of four; lifting them all costs 1 % of a step of 120 M bf16 parameters
__device__ inline void rounded_roots(const float* v, float* root) {
#pragma unroll
    for (int j = 0; j < 4; ++j) root[j] = root_step(v[j]);
    if (fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < kSmallMoment) {
#pragma unroll
        for (int j = 0; j < 4; ++j) root[j] = v[j] < kSmallMoment ? lifted_root(v[j]) : root[j];
    }
}
// a / b from y = 1 / b rounded to nearest
__device__ inline float rounded_quotient(float a, float b, float y) {
    const float q = a * y;
    return fmaf(fmaf(-q, b, a), y, q);
}
__device__ inline void moments_block(const Step& s, float g, float& m, float& v) {
    g *= s.scale;
    const float m0 = s.b1 * m, m1 = s.c1 * g;
    m = m0 + m1;
    const float v0 = s.b2 * v, v1 = (s.c2 * g) * g;
    v = v0 + v1;
}

// Largest finite magnitudes of a wave's first moments and second moments, and whether some are not finite.
__device__ inline uint32_t bits_of(float v) { return __float_as_uint(fabsf(v)); }
__device__ inline uint32_t finite_bits(float v) { return bits_of(v) < kInfinity ? bits_of(v) : 0u; }
__device__ inline bool block_tops(const float* me, const float* ve, float& top_m, float& top_v) {
    uint32_t a = max(max(bits_of(me[0]), bits_of(me[1])), max(bits_of(me[2]), bits_of(me[3])));
    uint32_t b = max(max(bits_of(ve[0]), bits_of(ve[1])), max(bits_of(ve[2]), bits_of(ve[3])));
    wave_max(a, b);
    const bool odd = max(a, b) >= kInfinity;
    if (odd) {
        a = max(max(finite_bits(me[0]), finite_bits(me[1])), max(finite_bits(me[2]), finite_bits(me[3])));
        b = max(max(finite_bits(ve[0]), finite_bits(ve[1])), max(finite_bits(ve[2]), finite_bits(ve[3])));
        wave_max(a, b);
    }
    top_m = __uint_as_float(a);
    top_v = __uint_as_float(b);
    return odd;
}
struct Scale {
    float s, y;                              // the scale and its reciprocal; both 0 where everything is
};
__device__ inline Scale scale_of(float top) {
    const float s = top * (1.f / kTopCode);
    const float y0 = __builtin_amdgcn_rcpf(s), y = fmaf(fmaf(-s, y0, 1.f), y0, y0);
    return s > kLeastScale ? Scale{s, y} : Scale{0.f, 0.f};
}
// A block's scales and codes from its moments: me and ve, root the roots of ve.  The conversion adds a word's upper 20 bits below the
// last bit that it keeps.
__device__ inline void codes_of(const float* me, const float* ve, const float* root, const uint32_t* words, uint32_t& cm, uint32_t& cr, float& ms, float& vs) {
    float top_m, top_v;
    const bool odd = block_tops(me, ve, top_m, top_v);
    const Scale a = scale_of(top_m), b = scale_of(rounded_root(top_v));
    ms = a.s;
    vs = b.s;
    float x[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[j] = __builtin_amdgcn_fmed3f(rounded_quotient(me[j], a.s, a.y), -kTopCode, kTopCode);
        const float q = rounded_quotient(root[j], b.s, b.y);
        y[j] = q > 0.f ? __builtin_amdgcn_fmed3f(q, kLeastCode, kTopCode) : 0.f;
    }
    if (odd) {                               // (the same for the whole wave)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = bits_of(me[j]) < kInfinity ? x[j] : __builtin_nanf("");
            y[j] = bits_of(ve[j]) < kInfinity ? y[j] : __builtin_nanf("");
        }
    }
    int p = 0, q = 0;
    p = __builtin_amdgcn_cvt_sr_fp8_f32(x[0], words[0], p, 0);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], words[0] << 16, q, 0);
    p = __builtin_amdgcn_cvt_sr_fp8_f32(x[1], words[1], p, 1);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], words[1] << 16, q, 1);
    p = __builtin_amdgcn_cvt_sr_fp8_f32(x[2], words[2], p, 2);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], words[2] << 16, q, 2);
    p = __builtin_amdgcn_cvt_sr_fp8_f32(x[3], words[3], p, 3);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], words[3] << 16, q, 3);
    cm = (uint32_t)p;
    cr = (uint32_t)q;
}
__device__ inline uint32_t block_key(const Step& s, int64_t lo) { return s.key ^ (uint32_t)(lo >> 32) * 0x9E3779B1u; }   // a block never crosses 2^32

// Which states the tensors of a call have: one kind alone takes fewer registers.
enum StateKinds { FLOAT_STATES = 1, BLOCK_STATES = 2, BOTH_STATES = 3 };
template <int KINDS>
__device__ inline bool has_blocks(const AdamTensor& t) { return KINDS == BLOCK_STATES || (KINDS == BOTH_STATES && t.state_type == LEGEND_STATE_BLOCK); }

// K whole blocks of 256 elements as a wave loads them, kApart elements from one to the next: four neighbouring elements a lane.
constexpr int kApart = 4 * kAdamBlock;
typedef uint32_t code_word __attribute__((aligned(1)));
template <int K, bool STREAM, int KINDS>
struct Blocks {
    uint4 g[K], p[K], m[K], v[K];            // 8-bit states: four codes in m.x and v.x, the block's scales in m.y and v.y

    __device__ void load(const AdamTensor& t, const void* grad, int64_t lo) {
        const int64_t i0 = lo + lane_id() * 4;
        const int ptype = t.master ? (int)LEGEND_TYPE_FLOAT : t.param_type;
        const void* from = t.master ? t.master : t.param;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            g[k] = raw_quad<false>(grad, i0 + k * kApart, t.grad_type);
            p[k] = raw_quad<STREAM>(from, i0 + k * kApart, ptype);
        }
        if (has_blocks<KINDS>(t)) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const code_word* cm = reinterpret_cast<const code_word*>(static_cast<const uint8_t*>(t.m) + i0 + k * kApart);
                const code_word* cv = reinterpret_cast<const code_word*>(static_cast<const uint8_t*>(t.v) + i0 + k * kApart);
                m[k].x = STREAM ? __builtin_nontemporal_load(cm) : *cm;
                v[k].x = STREAM ? __builtin_nontemporal_load(cv) : *cv;
                m[k].y = __float_as_uint(t.m_scale[lo / kAdamBlock + k * (kApart / kAdamBlock)]);
                v[k].y = __float_as_uint(t.v_scale[lo / kAdamBlock + k * (kApart / kAdamBlock)]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                m[k] = raw_quad<STREAM>(t.m, i0 + k * kApart, LEGEND_TYPE_FLOAT);
                v[k] = raw_quad<STREAM>(t.v, i0 + k * kApart, LEGEND_TYPE_FLOAT);
            }
        }
    }

    template <bool BLOCK>
    __device__ void finish(const AdamTensor& t, const Step& s, int64_t lo) const {
        const int ptype = t.master ? (int)LEGEND_TYPE_FLOAT : t.param_type;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t i = lo + lane_id() * 4 + k * kApart;
            float ge[4], pe[4], me[4], ve[4], root[4];
            numbers_of(g[k], t.grad_type, ge);
            numbers_of(p[k], ptype, pe);
            if (BLOCK) {
                codes_to_numbers(m[k].x, __uint_as_float(m[k].y), me);
                codes_to_numbers(v[k].x, __uint_as_float(v[k].y), ve);
#pragma unroll
                for (int j = 0; j < 4; ++j) ve[j] *= ve[j];
            } else {
                numbers_of(m[k], LEGEND_TYPE_FLOAT, me);
                numbers_of(v[k], LEGEND_TYPE_FLOAT, ve);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (BLOCK) moments_block(s, ge[j], me[j], ve[j]);
                else step_float(s, ge[j], me[j], ve[j], pe[j]);
            }
            if (BLOCK) {
                rounded_roots(ve, root);
#pragma unroll
                for (int j = 0; j < 4; ++j) pe[j] = step_parameter(s, me[j], root[j], pe[j]);
            }
            if (t.master) store_quad<STREAM>(t.master + i, pe);
            put_quad<STREAM>(t.param, i, t.param_type, pe);
            if (!BLOCK) {
                store_quad<STREAM>(static_cast<float*>(t.m) + i, me);
                store_quad<STREAM>(static_cast<float*>(t.v) + i, ve);
                continue;
            }
            const int64_t at = lo + k * kApart;
            const uint32_t key = block_key(s, at);
            const uint32_t words[4] = {random_word((uint32_t)i ^ key), random_word((uint32_t)(i + 1) ^ key),
                                       random_word((uint32_t)(i + 2) ^ key), random_word((uint32_t)(i + 3) ^ key)};
            uint32_t cm, cr;
            float ms, vs;
            codes_of(me, ve, root, words, cm, cr, ms, vs);
            code_word* to_m = reinterpret_cast<code_word*>(static_cast<uint8_t*>(t.m) + i);
            code_word* to_v = reinterpret_cast<code_word*>(static_cast<uint8_t*>(t.v) + i);
            if (STREAM) {
                __builtin_nontemporal_store(cm, to_m);
                __builtin_nontemporal_store(cr, to_v);
            } else {
                *to_m = cm;
                *to_v = cr;
            }
            if (lane_id() == 0) {
                t.m_scale[at / kAdamBlock] = ms;
                t.v_scale[at / kAdamBlock] = vs;
            }
        }
    }
    __device__ void any_finish(const AdamTensor& t, const Step& s, int64_t lo) const {
        if (has_blocks<KINDS>(t)) finish<true>(t, s, lo);
        else finish<false>(t, s, lo);
    }
};

// The last block of a tensor, elements [lo, count): single elements, neighbours in neighbouring lanes.
template <int KINDS>
__device__ inline void part_block(const AdamTensor& t, const void* grad, const Step& s, int64_t lo) {
    const bool block = has_blocks<KINDS>(t);
    const float ms = block ? t.m_scale[lo / kAdamBlock] : 1.f, vs = block ? t.v_scale[lo / kAdamBlock] : 1.f;
    float m[4], v[4], root[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = lo + j * kWave + lane_id();
        m[j] = v[j] = root[j] = 0.f;
        if (i >= t.count) continue;
        if (block) {
            m[j] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.m)[i], 0) * ms;
            v[j] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.v)[i], 0) * vs;
            v[j] *= v[j];
        } else {
            m[j] = static_cast<const float*>(t.m)[i];
            v[j] = static_cast<const float*>(t.v)[i];
        }
        float p = t.master ? t.master[i] : load_as(t.param, i, t.param_type);
        const float g = load_as(grad, i, t.grad_type);
        if (block) {
            moments_block(s, g, m[j], v[j]);
            root[j] = rounded_root(v[j]);
            p = step_parameter(s, m[j], root[j], p);
        } else {
            step_float(s, g, m[j], v[j], p);
        }
        if (t.master) t.master[i] = p;
        store_as(t.param, i, t.param_type, p);
        if (!block) {
            static_cast<float*>(t.m)[i] = m[j];
            static_cast<float*>(t.v)[i] = v[j];
        }
    }
    if (!block) return;
    const uint32_t key = block_key(s, lo);
    uint32_t words[4], cm, cr;
    float new_ms, new_vs;
#pragma unroll
    for (int j = 0; j < 4; ++j) words[j] = random_word((uint32_t)(lo + j * kWave + lane_id()) ^ key);
    codes_of(m, v, root, words, cm, cr, new_ms, new_vs);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = lo + j * kWave + lane_id();
        if (i >= t.count) continue;
        static_cast<uint8_t*>(t.m)[i] = (uint8_t)(cm >> (8 * j));
        static_cast<uint8_t*>(t.v)[i] = (uint8_t)(cr >> (8 * j));
    }
    if (lane_id() == 0) {
        t.m_scale[lo / kAdamBlock] = new_ms;
        t.v_scale[lo / kAdamBlock] = new_vs;
    }
}

// A wave's blocks of a unit that the tensor ends in.
template <int K, bool STREAM, int KINDS>
__device__ inline void part_unit(const AdamTensor& t, const void* grad, const Step& s, int64_t lo) {
    for (int k = 0; k < K; ++k) {
        const int64_t at = lo + k * kApart;
        if (at >= t.count) break;
        if (at + kAdamBlock > t.count) {
            part_block<KINDS>(t, grad, s, at);
        } else {
            Blocks<1, STREAM, KINDS> one;
            one.load(t, grad, at);
            one.any_finish(t, s, at);
        }
    }
}

// What a step reads of the state and what it leaves lie apart: a kernel before its last one (the squares', the one that finishes the
// norm, or one for this alone) makes the one from the other, its last writes the other.  No workgroup waits for another.  Only where
// there is no norm and few workgroups, the step is one launch (ALONE), and the workgroup that counts itself done last writes what all
// have read: by then every other has, and nothing else that one workgroup wrote is read by another, so that the counter needs no order
// of memory.  A count takes 10 ns, a launch 4 us.  (41 000 elements without a norm: 5.5 us, in two launches 8.3)
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

// What the gradients are multiplied by, from the partial sums; the same in all of 256 threads.
__device__ inline float gradient_scale(const AdamParams& a, int parts, double* box, bool reports, bool& skip) {
    float scale = a.grad_scale ? *a.grad_scale : 1.f;
    skip = false;
    if (!a.with_norm) return scale;
    double sum = 0.0;
    for (int k = threadIdx.x; k < parts; k += 256) sum += a.partial[k];
    const double norm = sqrt(block_sum(sum, box)) * fabs((double)scale);
    skip = !(norm < __builtin_inf());
    if (a.norm_out && reports) *a.norm_out = (float)norm;
    if (a.max_norm > 0.0 && norm > a.max_norm) scale = (float)(a.max_norm / (norm + 1e-6)) * scale;
    return scale;
}
__global__ void __launch_bounds__(256) k_finish_norm(AdamParams a, int parts) {
    __shared__ double box[4];
    bool skip;
    const float scale = gradient_scale(a, parts, box, threadIdx.x == 0, skip);
    if (threadIdx.x) return;
    begin_step(a);
    a.state->scale = scale;
    a.state->skip = skip ? 1u : 0u;
}

// K: blocks that a wave takes of a unit (unit_elems = 4 K blocks).
template <int K>
__global__ void __launch_bounds__(256) k_grad_squares(AdamParams a) {
    __shared__ double box[4];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (K == 1 && blockIdx.x == 0 && threadIdx.x == 0) begin_step(a);
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
            for (int k = 0; k < K; ++k) r[k] = raw_quad<false>(grad, lo + k * kApart + threadIdx.x * 4, type);
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

template <int K, bool STREAM, int KINDS, bool ALONE>
__global__ void __launch_bounds__(256) k_adamw(AdamParams a, int norm_parts) {
    __shared__ double box[4];
    const TensorTable tensors = (TensorTable)a.tensors;
    const UnitTable units = (UnitTable)a.unit_tensor;
    const GradTable grads = (GradTable)a.grads;
    double lr = 0.0, inv_bias1 = 0.0;
    uint64_t key = 0;
    Step s;
    bool ready = false, skip = false;
    AdamState read;                              // ALONE: as every workgroup finds it
    auto prepare = [&]() {
        ready = true;
        if (ALONE) {
            read = *a.state;
            inv_bias1 = 1.0 / (1.0 - read.power1);
            key = hash_fold(a.seed, (uint64_t)(read.steps + 1));
            s.inv_bias2_root = (float)(1.0 / sqrt(1.0 - read.power2));
        } else {
            inv_bias1 = a.state->inv_bias1;
            key = a.state->key;
            s.inv_bias2_root = a.state->inv_bias2_root;
        }
        if (K > 1) {
            s.scale = a.state->scale;
            skip = a.state->skip != 0;
        } else {
            s.scale = gradient_scale(a, norm_parts, box, blockIdx.x == 0 && threadIdx.x == 0, skip);
        }
        lr = a.lr * (a.lr_factor ? (double)*a.lr_factor : 1.0);
        constants_of(a, s);
    };
    for (int64_t u = blockIdx.x; u < a.units; u += gridDim.x) {
        const int k0 = units[u];
        const AdamTensor t = tensor_at(tensors + k0);
        const void* grad = grads[k0];
        const int64_t unit_lo = (u - t.first_unit) * (K * kApart), lo = unit_lo + (threadIdx.x / kWave) * kAdamBlock;
        const bool whole = unit_lo + K * kApart <= t.count;
        Blocks<K, STREAM, KINDS> in;
        if (whole) in.load(t, grad, lo);
        if (!ready) prepare();                   // the first unit's numbers are on their way meanwhile
        if (skip) break;
        rates_of(t, lr, inv_bias1, key, s);
        if (whole) in.any_finish(t, s, lo);
        else part_unit<K, STREAM, KINDS>(t, grad, s, lo);
    }
    if (!ready) prepare();                       // no units at all

    if (ALONE) {
        __syncthreads();
        if (threadIdx.x) return;
        if (__hip_atomic_fetch_add(&a.state->ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 < gridDim.x) return;
        a.state->ticket = 0;
        a.state->steps = read.steps + 1;
        a.state->power1 = read.power1 * a.beta1;
        a.state->power2 = read.power2 * a.beta2;
    } else if (blockIdx.x == 0 && threadIdx.x == 0) {
        AdamState& st = *a.state;
        st.steps = st.now_steps + (skip ? 0 : 1);
        st.skipped = st.now_skipped + (skip ? 1 : 0);
        st.power1 = st.now_power1 * (skip ? 1.0 : a.beta1);
        st.power2 = st.now_power2 * (skip ? 1.0 : a.beta2);
    }
}

int adam_unit_elems(int64_t total) { return total >= kLargeTotal ? 2 * kApart : kApart; }

void adam_state_at(AdamState* s, int64_t steps, double beta1, double beta2) {
    *s = AdamState{};
    s->steps = steps;
    s->power1 = std::pow(beta1, (double)(steps + 1));
    s->power2 = std::pow(beta2, (double)(steps + 1));
}

template <int K, bool STREAM, bool ALONE>
static void launch_step(hipStream_t st, const AdamParams& a, int64_t grid, int parts) {
    if (a.kinds == FLOAT_STATES) k_adamw<K, STREAM, FLOAT_STATES, ALONE><<<(unsigned)grid, 256, 0, st>>>(a, parts);
    else if (a.kinds == BLOCK_STATES) k_adamw<K, STREAM, BLOCK_STATES, ALONE><<<(unsigned)grid, 256, 0, st>>>(a, parts);
    else k_adamw<K, STREAM, BOTH_STATES, ALONE><<<(unsigned)grid, 256, 0, st>>>(a, parts);
}

template <int K, bool STREAM>
static hipError_t launch_units(hipStream_t st, const AdamParams& a) {
    const int64_t most_parts = K > 1 ? kPartsLarge : kPartsSmall;
    const int parts = (int)(a.units < most_parts ? a.units : most_parts);
    const bool squares = a.with_norm && parts > 0;
    const int64_t grid = adam_grid(a.units, K > 1);
    if constexpr (K == 1) {
        if (!a.with_norm && grid <= kGridAlone) {
            launch_step<K, STREAM, true>(st, a, grid, 0);
            return hipGetLastError();
        }
    }
    if (squares) k_grad_squares<K><<<parts, 256, 0, st>>>(a);
    if (K > 1) k_finish_norm<<<1, 256, 0, st>>>(a, parts);
    else if (!squares) k_begin_step<<<1, 1, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    launch_step<K, STREAM, false>(st, a, grid, parts);
    return hipGetLastError();
}

hipError_t launch_adamw(hipStream_t st, const AdamParams& a) {
    if (a.unit_elems == kApart) return launch_units<1, false>(st, a);
    return a.stream ? launch_units<2, true>(st, a) : launch_units<2, false>(st, a);
}

}  // namespace legend
