// One AdamW step over many tensors in one launch, and the norm of all their gradients.
//
//   g = grad * grad_scale * clip        m = b1 m + (1 - b1) g        v = b2 v + (1 - b2) g^2
//   w = w (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// The step is bound by HBM: with fp32 gradients and 16-bit weights 24 bytes a weight (fp32 states), 12 with states of
// 8 bits.  A plan in device memory lists the tensors and, for each chunk of 4096 weights, whose it is: the grid is the
// chunks of all tensors, so hundreds of small matrices fill the chip like one large one.
//
// 8-bit states.  256 consecutive weights share a scale, the power of two that brings the largest magnitude into
// (224, 448]; the codes are e4m3, which keeps four significant bits over 17 powers of two, and a power of two for a scale
// makes the rounding to a code the only one.  m is stored as it is and v as its square root: half the range.  Codes are
// rounded up or down at random with the odds of the value's place between them: with b2 = 0.999 a step moves v by less
// than half the distance of two codes, and rounding to nearest would never let it decay.  The random bits are a hash of
// the caller's seed, the step's number and the weight's place, so a run can be repeated bit by bit.  A second moment
// above zero keeps a code above zero: m / sqrt(v) stays bounded.
//
// Products and sums of the moments are rounded one by one (no fused multiply-add): a block's scale follows from its
// largest moment, and an implementation from the formulas in fp32 finds the same bits.
#include "../../include/qlora.h"
#include "common.hpp"
#include "kernels.hpp"

namespace qlora {

namespace {

constexpr int OT = 256;                      // threads of a workgroup
constexpr int CHUNK = OPTIM_CHUNK, PASSES = CHUNK / (OT * 4);
constexpr int QBLOCK = QLORA_OPTIM_BLOCK;    // weights that share a scale: one wave's four weights a lane
static_assert(QBLOCK == 4 * WAVE && CHUNK % QBLOCK == 0, "one wave, one block");

// odd words of the fractions of sqrt 2, sqrt 3 and the golden ratio
__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// four consecutive entries as they lie in memory: fp32 in four words, 16-bit in two; `have` of them exist, the rest are 0
__device__ __forceinline__ u32x4_t load4(const void *p, long i, int dtype, long have)
{
    u32x4_t r = {0, 0, 0, 0};
    if (dtype == QLORA_F32) {
        const uint32_t *f = (const uint32_t *)p + i;
        if (have >= 4)
            r = *(const u32x4_t *)f;
        else
            for (int e = 0; e < 3; ++e)
                if (e < have) r[e] = f[e];
    } else {
        const uint16_t *h = (const uint16_t *)p + i;
        if (have >= 4) {
            const u32x2_t v = *(const u32x2_t *)h;
            r[0] = v[0];
            r[1] = v[1];
        } else
            for (int e = 0; e < 3; ++e)
                if (e < have) r[e >> 1] |= (uint32_t)h[e] << (16 * (e & 1));
    }
    return r;
}
__device__ __forceinline__ void widen4(const u32x4_t &r, int dtype, float *f)
{
    if (dtype == QLORA_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(r[e]);
    } else if (dtype == QLORA_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = bf16_bits_to_f32((uint16_t)(r[e >> 1] >> (16 * (e & 1))));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = f16_bits_to_f32((uint16_t)(r[e >> 1] >> (16 * (e & 1))));
    }
}
__device__ __forceinline__ void store4(void *p, long i, int dtype, long have, const float *f)
{
    if (dtype == QLORA_F32) {
        float *d = (float *)p + i;
        if (have >= 4)
            *(float4_t *)d = float4_t{f[0], f[1], f[2], f[3]};
        else
            for (int e = 0; e < 3; ++e)
                if (e < have) d[e] = f[e];
    } else {
        uint16_t *d = (uint16_t *)p + i;
        u16x4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = dtype == QLORA_BF16 ? f32_to_bf16_bits(f[e]) : f32_to_f16_bits(f[e]);
        if (have >= 4)
            *(u16x4_t *)d = h;
        else
            for (int e = 0; e < 3; ++e)
                if (e < have) d[e] = h[e];
    }
}
__device__ __forceinline__ uint32_t load_codes(const void *p, long i, long have)
{
    const uint8_t *c = (const uint8_t *)p + i;
    if (have >= 4) return *(const uint32_t *)c;
    uint32_t r = 0;
    for (int e = 0; e < 3; ++e)
        if (e < have) r |= (uint32_t)c[e] << (8 * e);
    return r;
}
__device__ __forceinline__ void store_codes(void *p, long i, long have, uint32_t r)
{
    uint8_t *c = (uint8_t *)p + i;
    if (have >= 4)
        *(uint32_t *)c = r;
    else
        for (int e = 0; e < 3; ++e)
            if (e < have) c[e] = (uint8_t)(r >> (8 * e));
}
__device__ __forceinline__ void decode4(uint32_t codes, float scale, float *f)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    f[0] = lo[0] * scale;
    f[1] = lo[1] * scale;
    f[2] = hi[0] * scale;
    f[3] = hi[1] * scale;
}

// largest of the wave's values, as unsigned numbers (for bits of floats >= 0 the order of the floats; NaN above all)
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const uint32_t o = __shfl_xor(v, off, WAVE);
        v = v > o ? v : o;
    }
    return v;
}

// |x| <= 1.75 * 2^k, 0 <= r < 2^20: the e4m3 code of x / 2^(k - 8), rounded up where r exceeds the distance.  Multiplied by 2^-112
// (k taken off first) the code's exponent and mantissa are the top bits of the float, below the smallest normal code too.
__device__ __forceinline__ uint32_t encode(float x, int k, uint32_t r)
{
    const float y = fminf(ldexpf(fabsf(x), -112 - k), 1.75f * 0x1p-112f);
    return ((__float_as_uint(y) + r) >> 20) | (__float_as_uint(x) >> 31) << 7;
}

// the sum of the partial sums, the same in every thread of every workgroup
__device__ __forceinline__ double sum_parts(const double *__restrict__ parts, int count)
{
    __shared__ double red[OT / 64];
    double v = 0.0;
    for (int i = threadIdx.x; i < count; i += OT) v += parts[i];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, WAVE);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// what the coming step needs of the control block; nothing but this and the step's last lines writes there
__device__ __forceinline__ void prepare_step(qlora_optim_control_t *c, double beta1, double beta2)
{
    c->rate = (float)((double)c->lr / (1.0 - c->beta1_power * beta1));
    c->root = (float)(1.0 / sqrt(1.0 - c->beta2_power * beta2));
    c->key = mix(c->seed + (uint32_t)(c->step + 1) * 0x9E3779B9u);
}

__global__ void adamw_prepare_kernel(qlora_optim_control_t *c, double beta1, double beta2) { prepare_step(c, beta1, beta2); }

// parts[workgroup] = sum of the squares of its chunks' gradients, in 64 bits: no square leaves the range, and the sum of
// hundreds of millions of them keeps more than the 24 bits of the result
__global__ __launch_bounds__(OT) void grad_square_kernel(const OptimTensor *__restrict__ tensors,
                                                         const u32x2_t *__restrict__ table, uint32_t chunks,
                                                         double *parts, qlora_optim_control_t *control, double beta1,
                                                         double beta2)
{
    if (control && blockIdx.x == 0 && threadIdx.x == 0) prepare_step(control, beta1, beta2);
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const u32x2_t at = table[c];
        const OptimTensor *t = tensors + at[0];
        const int dtype = t->grad_dtype;
        const long first = (long)at[1] * CHUNK + threadIdx.x * 4, n = t->numel;
        u32x4_t g[PASSES];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) g[i] = load4(t->grad, first + i * OT * 4, dtype, n - first - i * OT * 4);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            float f[4];
            widen4(g[i], dtype, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = fma((double)f[e], (double)f[e], s);
        }
    }
    __shared__ double red[OT / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, WAVE);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) parts[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(OT) void grad_norm_kernel(const double *__restrict__ parts, int count, float grad_scale,
                                                       float *norm)
{
    const double s = sum_parts(parts, count);
    if (threadIdx.x == 0) norm[0] = (float)(sqrt(s) * fabs((double)grad_scale));
}

struct AdamArgs {
    const OptimTensor *tensors;
    const u32x2_t *table;
    qlora_optim_control_t *control;
    const double *parts;
    int count;                       // partial sums; 0: gradients are neither checked nor clipped
    double beta1, beta2, max_norm;
    float b1, c1, b2, c2, eps;       // beta, 1 - beta
};

struct AdamCoef {
    float gscale, decay, rate, root;
};

__device__ __forceinline__ void adam4(const AdamArgs &a, const AdamCoef &c, const float *g, float *m, float *v, float *u,
                                      float *w)
{
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = g[e] * c.gscale;
        m[e] = m[e] * a.b1 + x * a.c1;
        v[e] = v[e] * a.b2 + (x * x) * a.c2;
        u[e] = __builtin_amdgcn_sqrtf(v[e]);
        w[e] = w[e] * c.decay - c.rate * (m[e] * __builtin_amdgcn_rcpf(u[e] * c.root + a.eps));
    }
}

template <int BITS>
__device__ __forceinline__ void step_chunk(const AdamArgs &a, const OptimTensor &t, uint32_t chunk)
{
    const long first = (long)chunk * CHUNK + threadIdx.x * 4, n = t.numel;
    const bool master = t.master != nullptr;
    const int wide = master ? (int)QLORA_F32 : t.param_dtype;
    const void *wp = master ? (const void *)t.master : t.param;
    u32x4_t g[PASSES], w[PASSES], m[PASSES], v[PASSES];
    float ms[PASSES], vs[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const long at = first + i * OT * 4, have = n - at;
        g[i] = load4(t.grad, at, t.grad_dtype, have);
        w[i] = load4(wp, at, wide, have);
        if constexpr (BITS == 32) {
            m[i] = load4(t.exp_avg, at, QLORA_F32, have);
            v[i] = load4(t.exp_avg_sq, at, QLORA_F32, have);
        } else {
            m[i][0] = load_codes(t.exp_avg, at, have);
            v[i][0] = load_codes(t.exp_avg_sq, at, have);
            const long block = (at - (threadIdx.x & 63) * 4) / QBLOCK;         // the wave's
            ms[i] = block * QBLOCK < n ? t.avg_scale[block] : 0.f;
            vs[i] = block * QBLOCK < n ? t.avg_sq_scale[block] : 0.f;
        }
    }
    const qlora_optim_control_t *ctl = a.control;
    float gscale = ctl->grad_scale;
    if (a.count > 0) {
        const double norm = sqrt(sum_parts(a.parts, a.count)) * fabs((double)gscale);
        const bool finite = (float)norm < INFINITY;
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            a.control->grad_norm = (float)norm;
            if (!finite) a.control->skipped += 1;
        }
        if (!finite) return;                                                   // the step is not taken
        const double clip = a.max_norm / norm;
        gscale *= (float)(clip < 1.0 ? clip : 1.0);                            // (norm 0: no gradient to clip)
    }
    const AdamCoef c{gscale, 1.f - ctl->lr * t.lr_scale * t.weight_decay, ctl->rate * t.lr_scale, ctl->root};
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const long at = first + i * OT * 4, have = n - at;
        float gf[4], wf[4], mf[4], vf[4], uf[4];
        widen4(g[i], t.grad_dtype, gf);
        widen4(w[i], wide, wf);
        if constexpr (BITS == 32) {
            widen4(m[i], QLORA_F32, mf);
            widen4(v[i], QLORA_F32, vf);
        } else {
            decode4(m[i][0], ms[i], mf);
            decode4(v[i][0], vs[i], vf);
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[e] *= vf[e];
        }
        adam4(a, c, gf, mf, vf, uf, wf);
        if constexpr (BITS == 32) {
            if (have > 0) {
                store4(t.exp_avg, at, QLORA_F32, have, mf);
                store4(t.exp_avg_sq, at, QLORA_F32, have, vf);
            }
        } else {
            uint32_t mb = 0, vb = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t p = __float_as_uint(fabsf(mf[e])), q = __float_as_uint(vf[e]);
                mb = mb > p ? mb : p;
                vb = vb > q ? vb : q;
            }
            mb = wave_max_bits(mb);
            vb = wave_max_bits(vb);
            // 2^k: the largest |m| is at most 1.75 * 2^k, the largest v at most (1.75 * 2^k)^2 = 3.0625 * 4^k
            int km, kv;
            const float mf1 = frexpf(__uint_as_float(mb), &km);
            km = max(km - 1 + (mf1 > 0.875f), -126);
            const float vmax = __uint_as_float(vb);
            frexpf(vmax, &kv);
            kv = (kv - 1) >> 1;
            kv += ldexpf(vmax, -2 * kv) > 3.0625f;
            const long block = (at - (threadIdx.x & 63) * 4) / QBLOCK;
            const uint32_t place = (t.first_block + (uint32_t)block) * QBLOCK + (threadIdx.x & 63) * 4 + ctl->key;
            uint32_t mc = 0, vc = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t r = mix(place + e);
                mc |= encode(mf[e], km, r >> 12) << (8 * e);
                const uint32_t q = encode(uf[e], kv, r & 0xfffffu);
                vc |= (q == 0 && vf[e] > 0.f ? 1u : q) << (8 * e);
            }
            if (have > 0) {
                store_codes(t.exp_avg, at, have, mc);
                store_codes(t.exp_avg_sq, at, have, vc);
                if ((threadIdx.x & 63) == 0) {     // an infinity or a NaN makes NaN of the whole block
                    t.avg_scale[block] = mb == 0 ? 0.f : mb >= 0x7f800000u ? NAN : ldexpf(1.f, km - 8);
                    t.avg_sq_scale[block] = vb == 0 ? 0.f : vb >= 0x7f800000u ? NAN : ldexpf(1.f, kv - 8);
                }
            }
        }
        if (have > 0) {
            if (master) store4(t.master, at, QLORA_F32, have, wf);
            store4(t.param, at, t.param_dtype, have, wf);
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {             // no other workgroup reads these
        qlora_optim_control_t *w = a.control;
        w->step += 1;
        w->beta1_power *= a.beta1;
        w->beta2_power *= a.beta2;
    }
}

__global__ __launch_bounds__(OT) void adamw_kernel(const AdamArgs a)
{
    const u32x2_t at = a.table[blockIdx.x];
    const OptimTensor t = a.tensors[at[0]];
    if (t.state_bits == 8)
        step_chunk<8>(a, t, at[1]);
    else
        step_chunk<32>(a, t, at[1]);
}

inline const OptimTensor *tensors_of(const void *plan_device)
{
    return (const OptimTensor *)((const char *)plan_device + sizeof(OptimHeader));
}
inline const u32x2_t *table_of(const OptimHeader &h, const void *plan_device)
{
    return (const u32x2_t *)(tensors_of(plan_device) + h.count);
}

}  // namespace

void launch_grad_norm(const OptimHeader &h, const void *plan_device, float grad_scale, float *norm, double *parts,
                      hipStream_t s)
{
    const unsigned grid = h.chunks < OPTIM_PARTS ? h.chunks : OPTIM_PARTS;
    if (grid > 0)
        QLORA_LAUNCH(grad_square_kernel, dim3(grid), dim3(OT), 0, s, tensors_of(plan_device), table_of(h, plan_device),
                     h.chunks, parts, (qlora_optim_control_t *)nullptr, 0.0, 0.0);
    QLORA_LAUNCH(grad_norm_kernel, dim3(1), dim3(OT), 0, s, parts, (int)grid, grad_scale, norm);
}

void launch_adamw(const OptimHeader &h, const void *plan_device, void *control, double beta1, double beta2, double eps,
                  double max_norm, double *parts, hipStream_t s)
{
    qlora_optim_control_t *c = (qlora_optim_control_t *)control;
    const unsigned grid = h.chunks < OPTIM_PARTS ? h.chunks : OPTIM_PARTS;
    const bool guarded = max_norm > 0.0;
    if (guarded)
        QLORA_LAUNCH(grad_square_kernel, dim3(grid), dim3(OT), 0, s, tensors_of(plan_device), table_of(h, plan_device),
                     h.chunks, parts, c, beta1, beta2);
    else
        QLORA_LAUNCH(adamw_prepare_kernel, dim3(1), dim3(1), 0, s, c, beta1, beta2);
    const AdamArgs a{tensors_of(plan_device), table_of(h, plan_device), c, parts, guarded ? (int)grid : 0, beta1, beta2,
                     max_norm, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps};
    QLORA_LAUNCH(adamw_kernel, dim3(h.chunks), dim3(OT), 0, s, a);
}

}  // namespace qlora
