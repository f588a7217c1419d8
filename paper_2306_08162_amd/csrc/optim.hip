// One AdamW step over many tensors in one launch, and the norm of all their gradients.
//
//   g = grad * grad_scale * clip        m = b1 m + (1 - b1) g        v = b2 v + (1 - b2) g^2
//   w = w (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// The step is bound by HBM: with fp32 gradients and 16-bit weights 24 bytes a weight (fp32 states), 12 with states of
// 8 bits, and 4 more for the norm.  20M weights with fp32 masters: 103 us with the norm, 5.8 TB/s of the 600 MB that a step
// cannot do without (a large copy reaches 4.9 to 5.7); 160M with 8-bit states: 434 us, 5.9 TB/s with the second reading of the
// gradients counted, and 62 instructions a weight close behind it.
// A plan in device memory has a record for each chunk of up to 2048 weights of a tensor, one workgroup's work: hundreds of small
// matrices fill the chip like one large one.  (Chunks of 1024 and 4096: 517 and 481 us where 2048 took 485 on those 160M, but 22.3
// and 25.8 where it took 22.1 on 5M in 96 tensors.)
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

#include <cfloat>

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

// Device memory by type: a pointer read from the plan would otherwise be taken for one into any memory, with slower loads.
// ONCE: past the caches.  A step touches each of its bytes once, and whatever ran since the step before has replaced them:
// with the hint 448 fp32-state tensors of 600 MB take 103 us instead of 124, 37 MB 10.4 instead of 13.5 (3 to 11 % more
// only where steps of up to 225 MB follow one another with nothing in between).  The gradients' first reading, for their norm,
// leaves them in the caches.
template <bool ONCE, typename T>
__device__ __forceinline__ T load_global(const void *p, uint32_t byte)
{
    typedef const T __attribute__((address_space(1))) global_t;
    global_t *const at = (global_t *)((uintptr_t)p + byte);
    if constexpr (ONCE)
        return __builtin_nontemporal_load(at);
    else
        return *at;
}
template <typename T>
__device__ __forceinline__ void store_once(void *p, uint32_t byte, T v)
{
    typedef T __attribute__((address_space(1))) global_t;
    __builtin_nontemporal_store(v, (global_t *)((uintptr_t)p + byte));
}

// Entries [i, i + 4) of a chunk that begins at p and has `have` of them (FULL: all of CHUNK), as they lie in memory: fp32 in
// four words, 16-bit ones in two; those that do not exist are 0 and are not stored.
template <bool FULL, bool ONCE>
__device__ __forceinline__ u32x4_t load4(const void *p, uint32_t i, int dtype, uint32_t have)
{
    u32x4_t r = {0, 0, 0, 0};
    if (dtype == QLORA_F32) {
        if (FULL || i + 4 <= have)
            r = load_global<ONCE, u32x4_t>(p, 4 * i);
        else
            for (uint32_t e = 0; e < 3; ++e)
                if (i + e < have) r[e] = load_global<ONCE, uint32_t>(p, 4 * (i + e));
    } else {
        if (FULL || i + 4 <= have) {
            const u32x2_t v = load_global<ONCE, u32x2_t>(p, 2 * i);
            r[0] = v[0];
            r[1] = v[1];
        } else
            for (uint32_t e = 0; e < 3; ++e)
                if (i + e < have) r[e >> 1] |= (uint32_t)load_global<ONCE, uint16_t>(p, 2 * (i + e)) << (16 * (e & 1));
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
template <bool FULL>
__device__ __forceinline__ void store4(void *p, uint32_t i, int dtype, uint32_t have, const float *f)
{
    if (dtype == QLORA_F32) {
        if (FULL || i + 4 <= have)
            store_once(p, 4 * i, float4_t{f[0], f[1], f[2], f[3]});
        else
            for (uint32_t e = 0; e < 3; ++e)
                if (i + e < have) store_once(p, 4 * (i + e), f[e]);
    } else {
        u16x4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = dtype == QLORA_BF16 ? f32_to_bf16_bits(f[e]) : f32_to_f16_bits(f[e]);
        if (FULL || i + 4 <= have)
            store_once(p, 2 * i, h);
        else
            for (uint32_t e = 0; e < 3; ++e)
                if (i + e < have) store_once(p, 2 * (i + e), (uint16_t)h[e]);
    }
}
template <bool FULL>
__device__ __forceinline__ uint32_t load_codes(const void *p, uint32_t i, uint32_t have)
{
    if (FULL || i + 4 <= have) return load_global<true, uint32_t>(p, i);
    uint32_t r = 0;
    for (uint32_t e = 0; e < 3; ++e)
        if (i + e < have) r |= (uint32_t)load_global<true, uint8_t>(p, i + e) << (8 * e);
    return r;
}
template <bool FULL>
__device__ __forceinline__ void store_codes(void *p, uint32_t i, uint32_t have, uint32_t r)
{
    if (FULL || i + 4 <= have)
        store_once(p, i, r);
    else
        for (uint32_t e = 0; e < 3; ++e)
            if (i + e < have) store_once(p, i + e, (uint8_t)(r >> (8 * e)));
}
__device__ __forceinline__ void decode4(uint32_t codes, float scale, float *f)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    f[0] = lo[0] * scale;
    f[1] = lo[1] * scale;
    f[2] = hi[0] * scale;
    f[3] = hi[1] * scale;
}

// largest of the wave's values, as unsigned numbers (for bits of floats >= 0 the order of the floats; NaN above all): lane 63
// gathers it along rows of 16 lanes and from row to row
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
    return v > o ? v : o;
}
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v)
{
    v = max_dpp<0x111, 0xf>(v);
    v = max_dpp<0x112, 0xf>(v);
    v = max_dpp<0x114, 0xf>(v);
    v = max_dpp<0x118, 0xf>(v);
    v = max_dpp<0x142, 0xa>(v);
    v = max_dpp<0x143, 0xc>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// The smallest k >= -126 with x <= 1.75 * 2^k for the float x > 0 of these bits: its exponent, one more where the mantissa
// exceeds 0x600000.
__device__ __forceinline__ int scale_of(uint32_t bits)
{
    const int k = (int)((bits + 0x1fffffu) >> 23) - 127;
    return k > -126 ? k : -126;
}
// The smallest k with x <= (1.75 * 2^k)^2 = 3.0625 * 4^k: half of the exponent, rounded down, after one more where the
// mantissa exceeds 0x440000 (1.53125; of an even exponent that changes nothing).
__device__ __forceinline__ int root_scale_of(uint32_t bits)
{
    int b = (int)bits;
    if (b < 0x00800000) {                      // a number below the smallest normal one: as if there were exponents below 0
        const int top = 31 - __builtin_clz(bits | 1u);
        b = (b << (23 - top)) - 0x00800000 + (top - 22) * 0x00800000;
    }
    return ((((b + 0x3bffff) >> 23) - 127) >> 1);
}

// |x| <= 1.75 * 2^k, 0 <= r < 2^20: the e4m3 code of x / 2^(k - 8), rounded up where r exceeds the distance, in the top byte.
// Multiplied by 2^-112 (k taken off first) the code's exponent and mantissa are bits 26..20 of the float, below the smallest
// normal code too; what is under them does not matter.
__device__ __forceinline__ uint32_t encode(float x, int k, uint32_t r)
{
    const uint32_t y = __float_as_uint(ldexpf(fabsf(x), -112 - k));
    return (((y + r) << 4) & 0x7fffffffu) | (__float_as_uint(x) & 0x80000000u);
}
// The same for u = sqrt(v), which the hardware may leave one unit above 1.75 * 2^k; at least code 1 where v > 0.
__device__ __forceinline__ uint32_t encode_root(float u, float v, int k, uint32_t r)
{
    const uint32_t y = __float_as_uint(fminf(ldexpf(u, -112 - k), 1.75f * 0x1p-112f)) + r, least = v > 0.f ? 1u << 20 : 0u;
    return (y > least ? y : least) << 4;
}
// the top bytes of four words as one word
__device__ __forceinline__ uint32_t top_bytes(const uint32_t *t)
{
    return __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0703u) | __builtin_amdgcn_perm(t[3], t[2], 0x07030c0cu);
}

// the sum over a wave, in every lane
template <int CTRL, int ROWS>
__device__ __forceinline__ double add_dpp(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, false),
                   hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xf, false);
    return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum_f64(double v)
{
    v = add_dpp<0x111, 0xf>(v);
    v = add_dpp<0x112, 0xf>(v);
    v = add_dpp<0x114, 0xf>(v);
    v = add_dpp<0x118, 0xf>(v);
    v = add_dpp<0x142, 0xa>(v);
    v = add_dpp<0x143, 0xc>(v);
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63),
                   hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// A lane's share of the partial sums, and the sum of all of them in every lane of a wave.  A workgroup's first wave asks for
// its share before anything else, and adds while its chunk is on the way.
struct Parts {
    double v[OPTIM_PARTS / WAVE];
};
__device__ __forceinline__ Parts load_parts(const double *__restrict__ parts, int count)
{
    Parts p;
#pragma unroll
    for (int i = 0; i < (int)(OPTIM_PARTS / WAVE); ++i) {
        const int at = i * WAVE + (threadIdx.x & 63);
        p.v[i] = at < count ? parts[at] : 0.0;
    }
    return p;
}
__device__ __forceinline__ double sum_parts(const Parts &p)
{
    double v = p.v[0];
#pragma unroll
    for (int i = 1; i < (int)(OPTIM_PARTS / WAVE); ++i) v += p.v[i];
    return wave_sum_f64(v);
}

// what the coming step needs of the control block
struct Coming {
    float rate, root;
    uint32_t key;
};
__device__ __forceinline__ Coming coming_step(const qlora_optim_control_t *c, double beta1, double beta2)
{
    return Coming{(float)((double)c->lr / (1.0 - c->beta1_power * beta1)), (float)(1.0 / sqrt(1.0 - c->beta2_power * beta2)),
                  mix(c->seed + (uint32_t)(c->step + 1) * 0x9E3779B9u)};
}
__device__ __forceinline__ void prepare_step(qlora_optim_control_t *c, double beta1, double beta2)
{
    const Coming n = coming_step(c, beta1, beta2);
    c->rate = n.rate;
    c->root = n.root;
    c->key = n.key;
}
__device__ __forceinline__ void commit_step(qlora_optim_control_t *c, double beta1, double beta2)
{
    c->step += 1;
    c->beta1_power *= beta1;
    c->beta2_power *= beta2;
}

__global__ void adamw_prepare_kernel(qlora_optim_control_t *c, double beta1, double beta2) { prepare_step(c, beta1, beta2); }

// parts[workgroup] = sum of the squares of its chunks' gradients, in 64 bits: no square leaves the range, and the sum of
// hundreds of millions of them keeps more than the 24 bits of the result.  Each quarter of a workgroup has chunks of its own.
// One workgroup a compute unit and no more: every workgroup of the step reads all partial sums (with 1024 of them that
// was as much traffic as the gradients of 160 million weights).
constexpr int ST = 4 * OT;
__global__ __launch_bounds__(ST) void grad_square_kernel(const OptimChunk *__restrict__ table, uint32_t chunks,
                                                         double *parts, qlora_optim_control_t *control, double beta1,
                                                         double beta2)
{
    if (control && blockIdx.x == 0 && threadIdx.x == 0) prepare_step(control, beta1, beta2);
    const uint32_t quarter = __builtin_amdgcn_readfirstlane(threadIdx.x / OT), tid = threadIdx.x & (OT - 1);
    // whose chunk is next is found out while this one's gradients are on their way
    struct Place {
        const void *grad;
        uint32_t have;
        int dtype;
    };
    const auto place = [&](uint32_t c) { return Place{table[c].grad, table[c].weights, table[c].grad_dtype}; };
    double s = 0.0;
    uint32_t c = blockIdx.x + quarter * gridDim.x;
    Place next{};
    if (c < chunks) next = place(c);
    while (c < chunks) {
        const Place now = next;
        u32x4_t g[PASSES];
        if (now.have == CHUNK) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) g[i] = load4<true, false>(now.grad, (i * OT + tid) * 4, now.dtype, CHUNK);
        } else {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) g[i] = load4<false, false>(now.grad, (i * OT + tid) * 4, now.dtype, now.have);
        }
        c += 4 * gridDim.x;
        if (c < chunks) next = place(c);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            float f[4];
            widen4(g[i], now.dtype, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = fma((double)f[e], (double)f[e], s);
        }
    }
    __shared__ double red[ST / 64];
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x < 64) {
        s = wave_sum_f64(threadIdx.x < ST / 64 ? red[threadIdx.x] : 0.0);
        if (threadIdx.x == 0) parts[blockIdx.x] = s;
    }
}

__global__ __launch_bounds__(WAVE) void grad_norm_kernel(const double *__restrict__ parts, int count, float grad_scale,
                                                       float *norm)
{
    const double s = sum_parts(load_parts(parts, count));
    if (threadIdx.x == 0) norm[0] = (float)(sqrt(s) * fabs((double)grad_scale));
}

struct AdamArgs {
    const OptimChunk *table;
    qlora_optim_control_t *control;
    const double *parts;
    int count;                       // partial sums; 0: gradients are neither checked nor clipped
    double beta1, beta2, max_norm;
    float b1, c1, b2, c2, eps;       // beta, 1 - beta
};

struct AdamCoef {
    float gscale, decay, rate, root;
};

// m = its old value times b1 on the way in
__device__ __forceinline__ void adam4(const AdamArgs &a, const AdamCoef &c, const float *g, float *m, float *v, float *u,
                                      float *w)
{
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = g[e] * c.gscale;
        m[e] = m[e] + x * a.c1;
        v[e] = v[e] * a.b2 + (x * x) * a.c2;
        u[e] = __builtin_amdgcn_sqrtf(v[e]);
    }
    // the hardware's root takes what is below the smallest normal number for 0: those are brought up by a power of four first (a
    // test of four weights together: few waves have such a v, and one of zeros alone finds zeros again)
    if (fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < FLT_MIN) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (v[e] < FLT_MIN) u[e] = __builtin_amdgcn_sqrtf(v[e] * 0x1p64f) * 0x1p-32f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        w[e] = w[e] * c.decay - c.rate * (m[e] * __builtin_amdgcn_rcpf(u[e] * c.root + a.eps));
}

// ALONE: this launch is the whole step (see adamw_alone_kernel)
template <int BITS, bool FULL, bool ALONE>
__device__ __forceinline__ void step_chunk(const AdamArgs &a, const OptimChunk &t, const Parts &parts)
{
    const uint32_t have = FULL ? CHUNK : t.weights;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const bool master = t.master != nullptr;
    const int wide = master ? (int)QLORA_F32 : t.param_dtype, grad_dtype = t.grad_dtype, param_dtype = t.param_dtype;
    void *const main = master ? t.master : t.param;
    u32x4_t g[PASSES], w[PASSES], m[PASSES], v[PASSES];
    float ms[PASSES], vs[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const uint32_t at = (i * OT + threadIdx.x) * 4;
        g[i] = load4<FULL, true>(t.grad, at, grad_dtype, have);
        w[i] = load4<FULL, true>(main, at, wide, have);
        if constexpr (BITS == 32) {
            m[i] = load4<FULL, true>(t.exp_avg, at, QLORA_F32, have);
            v[i] = load4<FULL, true>(t.exp_avg_sq, at, QLORA_F32, have);
        } else {
            const uint32_t block = i * (OT / 64) + wave;               // the wave's
            const bool some = FULL || block * QBLOCK < have;
            m[i][0] = load_codes<FULL>(t.exp_avg, at, have);
            v[i][0] = load_codes<FULL>(t.exp_avg_sq, at, have);
            ms[i] = some ? load_global<true, float>(t.avg_scale, 4 * block) : 0.f;
            vs[i] = some ? load_global<true, float>(t.avg_sq_scale, 4 * block) : 0.f;
        }
    }
    const qlora_optim_control_t *ctl = a.control;
    float gscale = ctl->grad_scale;
    const float lr = ctl->lr;
    Coming now;
    if constexpr (ALONE) {
        __shared__ Coming shared;
        if (threadIdx.x == 0) {
            now = coming_step(ctl, a.beta1, a.beta2);
            shared = now;
            // what the commit changes has been read (here alone): the values are there before the arrival is counted
            asm volatile("" : : "v"(now.rate), "v"(now.root), "v"(now.key) : "memory");
            qlora_optim_control_t *w = a.control;
            if (__hip_atomic_fetch_add(&w->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
                w->arrived = 0;                                        // every workgroup has
                w->rate = now.rate;
                w->root = now.root;
                w->key = now.key;
                commit_step(w, a.beta1, a.beta2);
            }
        }
        __syncthreads();
        now = shared;
    } else {
        now = Coming{ctl->rate, ctl->root, ctl->key};
    }
    const float rate = now.rate * t.lr_scale, root = now.root;
    const uint32_t key = now.key + t.place + lane * 4;
    if (!ALONE && a.count > 0) {
        __shared__ float clipped;                                      // NaN: the step is not taken
        if (wave == 0) {
            const double norm = sqrt(sum_parts(parts)) * fabs((double)gscale), clip = a.max_norm / norm;
            // what is left of a gradient after clipping is at most min(norm, max_norm): its square has to stay in fp32
            const bool finite = (float)norm < INFINITY && (norm < 0x1p63 || a.max_norm < 0x1p63);
            if (lane == 0) clipped = finite ? gscale * (float)(clip < 1.0 ? clip : 1.0) : NAN;     // (norm 0: nothing to clip)
            if (blockIdx.x == 0 && lane == 0) {
                a.control->grad_norm = (float)norm;
                if (!finite) a.control->skipped += 1;
            }
        }
        __syncthreads();
        gscale = clipped;
        if (gscale != gscale) return;
    }
    const AdamCoef c{gscale, 1.f - lr * t.lr_scale * t.weight_decay, rate, root};
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const uint32_t at = (i * OT + threadIdx.x) * 4;
        float gf[4], wf[4], mf[4], vf[4], uf[4];
        widen4(g[i], grad_dtype, gf);
        widen4(w[i], wide, wf);
        if constexpr (BITS == 32) {
            widen4(m[i], QLORA_F32, mf);
            widen4(v[i], QLORA_F32, vf);
#pragma unroll
            for (int e = 0; e < 4; ++e) mf[e] *= a.b1;
        } else {
            decode4(m[i][0], ms[i] * a.b1, mf);                        // a power of two times b1: one rounding, as in 32 bits
            decode4(v[i][0], vs[i], vf);
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[e] *= vf[e];
        }
        adam4(a, c, gf, mf, vf, uf, wf);
        if constexpr (BITS == 32) {
            store4<FULL>(t.exp_avg, at, QLORA_F32, have, mf);
            store4<FULL>(t.exp_avg_sq, at, QLORA_F32, have, vf);
        } else {
            const uint32_t mb = wave_max_bits(__float_as_uint(
                fmaxf(fmaxf(fabsf(mf[0]), fabsf(mf[1])), fmaxf(fabsf(mf[2]), fabsf(mf[3])))));
            uint32_t vb = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) vb = vb > __float_as_uint(vf[e]) ? vb : __float_as_uint(vf[e]);
            vb = wave_max_bits(vb);
            const int km = scale_of(mb), kv = root_scale_of(vb);
            const uint32_t block = i * (OT / 64) + wave;
            uint32_t mc[4], vc[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t r = mix(key + block * QBLOCK + e);
                mc[e] = encode(mf[e], km, r >> 12);
                vc[e] = encode_root(uf[e], vf[e], kv, r & 0xfffffu);
            }
            store_codes<FULL>(t.exp_avg, at, have, top_bytes(mc));
            store_codes<FULL>(t.exp_avg_sq, at, have, top_bytes(vc));
            // A gradient that is not finite leaves v so too, and makes NaN of the whole block (m of a NaN alone shows nothing: the
            // maximum passes over it).
            const bool bad = vb >= 0x7f800000u;
            if (lane == 0 && (FULL || block * QBLOCK < have)) {
                store_once(t.avg_scale, 4 * block, bad ? NAN : mb == 0 ? 0.f : ldexpf(1.f, km - 8));
                store_once(t.avg_sq_scale, 4 * block, bad ? NAN : vb == 0 ? 0.f : ldexpf(1.f, kv - 8));
            }
        }
        if (master) store4<FULL>(main, at, QLORA_F32, have, wf);
        store4<FULL>(t.param, at, param_dtype, have, wf);
    }
    if (!ALONE && blockIdx.x == 0 && threadIdx.x == 0)     // no other workgroup reads these
        commit_step(a.control, a.beta1, a.beta2);
}

template <bool ALONE>
__device__ __forceinline__ void step_any(const AdamArgs &a, const Parts &parts)
{
    const OptimChunk t = a.table[blockIdx.x];
    const bool full = t.weights == CHUNK;
    if (t.state_bits == 8) {
        if (full)
            step_chunk<8, true, ALONE>(a, t, parts);
        else
            step_chunk<8, false, ALONE>(a, t, parts);
    } else {
        if (full)
            step_chunk<32, true, ALONE>(a, t, parts);
        else
            step_chunk<32, false, ALONE>(a, t, parts);
    }
}

// Six waves a SIMD: five to seven are alike, with eight (which fewer registers would allow) the 448 fp32-state tensors take 117 us
// instead of 103: more streams at once than the memory keeps open.
__global__ __launch_bounds__(OT) __attribute__((amdgpu_waves_per_eu(6, 6))) void adamw_kernel(const AdamArgs a)
{
    Parts parts{};
    if (a.count > 0 && threadIdx.x < WAVE) parts = load_parts(a.parts, a.count);
    step_any<false>(a, parts);
}

// A small step without clipping, in one launch: each workgroup works out the coming step for itself while its chunk is on the
// way, and the last one to have read the control block commits.  Their arrivals are counted in the control block, one after
// the other, 13 ns each: 64 chunks take 4.5 us (8-bit states 5.3) where two launches take 7.0 (6.9), 128 take 5.1 (6.0), but 256
// 6.7 (7.5) and 512 10.4 (10.9) where those take 6.8 (6.8) and 7.1 (7.3).
constexpr uint32_t ALONE_CHUNKS = 128;
__global__ __launch_bounds__(OT) void adamw_alone_kernel(const AdamArgs a) { step_any<true>(a, Parts{}); }

inline const OptimChunk *table_of(const void *plan_device)
{
    return (const OptimChunk *)((const char *)plan_device + sizeof(OptimHeader));
}
inline unsigned square_grid(const OptimHeader &h) { return h.chunks < OPTIM_PARTS ? h.chunks : OPTIM_PARTS; }

}  // namespace

void launch_grad_norm(const OptimHeader &h, const void *plan_device, float grad_scale, float *norm, double *parts,
                      hipStream_t s)
{
    const unsigned grid = square_grid(h);
    QLORA_LAUNCH(grad_square_kernel, dim3(grid), dim3(ST), 0, s, table_of(plan_device), h.chunks, parts,
                 (qlora_optim_control_t *)nullptr, 0.0, 0.0);
    QLORA_LAUNCH(grad_norm_kernel, dim3(1), dim3(WAVE), 0, s, parts, (int)grid, grad_scale, norm);
}

void launch_adamw(const OptimHeader &h, const void *plan_device, void *control, double beta1, double beta2, double eps,
                  double max_norm, double *parts, hipStream_t s)
{
    qlora_optim_control_t *c = (qlora_optim_control_t *)control;
    const unsigned grid = square_grid(h);
    const bool guarded = max_norm > 0.0;
    const AdamArgs a{table_of(plan_device), c, parts, guarded ? (int)grid : 0, beta1, beta2,
                     max_norm, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps};
    if (!guarded && h.chunks <= ALONE_CHUNKS) {
        QLORA_LAUNCH(adamw_alone_kernel, dim3(h.chunks), dim3(OT), 0, s, a);
        return;
    }
    if (guarded)
        QLORA_LAUNCH(grad_square_kernel, dim3(grid), dim3(ST), 0, s, table_of(plan_device), h.chunks, parts, c, beta1, beta2);
    else
        QLORA_LAUNCH(adamw_prepare_kernel, dim3(1), dim3(1), 0, s, c, beta1, beta2);
    QLORA_LAUNCH(adamw_kernel, dim3(h.chunks), dim3(OT), 0, s, a);
}

}  // namespace qlora
