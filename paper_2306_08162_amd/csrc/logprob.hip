// Log probabilities of given tokens, the entropy and the most likely alternatives of each row of logits, and the
// gradient of the first two with respect to the logits.
//
//   m = max z,  S = sum_i exp(z_i - m),   log p_i = (z_i - m) - ln S
//   entropy   H = -sum_i p_i log p_i = ln S + sum_i exp(z_i - m) (m - z_i) / S
//   gradient  of g log p_t + h H:   dz_i = g [i = t] - p_i (g + h (log p_i + H))
//
// The work is bound by HBM: a row is read once (and, backward, once more and its gradient written).  One workgroup takes
// up to 64 KB of a row into registers, so the maximum is known before the first exponential and no sum is ever rescaled;
// longer rows, and rows too few to fill the chip, are cut into segments whose results a second launch joins.
//
// A token that is almost certain has p = 1 / (1 + s) with a tiny s, and S = 1 + s would round it away: the sums keep
// the entries equal to the maximum as a count n apart from the sum s of all others, ln S = log1p(s) where n = 1, and
// log p and H of such a row keep their relative accuracy.
//
// Alternatives.  The threads of a workgroup form g >= k groups; every group's largest entry is at least
// tau = the smallest of the g maxima, so at least k entries are >= tau and, on rows in no special order, not many more
// than g ln g: they are collected in LDS as 64-bit keys (value, lower index first) and sorted by waves.  Rows that break
// the rule of thumb (an ordered vocabulary, masks of the type's lowest number) take exact detours: the threshold is
// raised by bisection until the entries above it fit, and entries equal to it are taken in order of their index.
#include "common.hpp"
#include "kernels.hpp"

namespace qlora {

namespace {

constexpr int PT = 512;              // most threads of a workgroup
constexpr int PCH = 8;               // 16-byte pieces a thread holds
constexpr int PCAP = 1024;           // keys that LDS holds
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// x log2 of a weight that is zero: far below what exp2 can represent, and finite, so that 0 * x stays 0
constexpr float NOTHING = -1024.f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

struct ScoreArgs {
    const void *z;
    long stride;                     // elements from row to row
    const int32_t *token;
    float *logprob, *entropy;
    int32_t *alt_token;
    float *alt_logprob;
    float4_t *stats;
    int M, V, k;
    int splits, seg;                 // segments of a row, 16-byte pieces of a segment
    float4_t *part;                  // [M, splits]: m, n, s, q
    unsigned long long *lists;       // [M, splits, k]
};

// rows start at any element: 16-byte accesses with the alignment of an element
typedef u32x4_t __attribute__((aligned(2))) loose_t;

// DT: 0 fp16, 1 bf16, 2 fp32
template <int DT>
struct Piece {
    static constexpr int E = DT == 2 ? 4 : 8;
    u32x4_t w;
    __device__ __forceinline__ float val(int e) const
    {
        if constexpr (DT == 2) return __uint_as_float(w[e]);
        if constexpr (DT == 1) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        return (float)__builtin_bit_cast(half8_t, w)[e];
    }
    __device__ __forceinline__ float max() const
    {
        if constexpr (DT == 0) {
            const half8_t h = __builtin_bit_cast(half8_t, w);
            const half2_t a = {h[0], h[1]}, b = {h[2], h[3]}, c = {h[4], h[5]}, d = {h[6], h[7]};
            const half2_t v = __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d));
            return fmaxf((float)v[0], (float)v[1]);
        } else {
            float v = val(0);
#pragma unroll
            for (int e = 1; e < E; ++e) v = fmaxf(v, val(e));
            return v;
        }
    }
    // entries [0, have) of a row's last piece; the rest are -inf, which weighs nothing and is no alternative
    __device__ __forceinline__ void load_part(const void *row, long at, int have)
    {
        if constexpr (DT == 2) {
            const uint32_t *p = (const uint32_t *)row + at;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = e < have ? p[e] : 0xff800000u;
        } else {
            const uint16_t *p = (const uint16_t *)row + at;
            constexpr uint32_t ninf = DT == 1 ? 0xff80u : 0xfc00u;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t lo = e < have ? p[e] : ninf, hi = e + 1 < have ? p[e + 1] : ninf;
                w[e >> 1] = lo | hi << 16;
            }
        }
    }
};

// order of the floats as unsigned numbers (-0 counts as 0), and back
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o)
{
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
constexpr uint32_t ORDER_NINF = 0x007fffffu;           // order_of(-inf)

typedef unsigned long long key_t;                      // order << 32 | ~index: larger is better, 0 is nothing

__device__ __forceinline__ key_t shfl_key(key_t v, int from)
{
    const uint32_t lo = __shfl((uint32_t)v, from, WAVE), hi = __shfl((uint32_t)(v >> 32), from, WAVE);
    return (key_t)hi << 32 | lo;
}
__device__ __forceinline__ key_t exchange(key_t v, int lane, int stride, bool descending)
{
    const key_t o = shfl_key(v, lane ^ stride);
    return ((lane & stride) == 0) == descending ? (v > o ? v : o) : (v > o ? o : v);
}
// the wave's 64 keys in descending order over the lanes (bitonic)
__device__ __forceinline__ key_t sort64(key_t v, int lane)
{
    for (int size = 2; size <= 64; size <<= 1)
        for (int stride = size >> 1; stride > 0; stride >>= 1) v = exchange(v, lane, stride, (lane & size) == 0);
    return v;
}
// the 64 largest of two descending lists
__device__ __forceinline__ key_t merge64(key_t a, key_t b, int lane)
{
    const key_t r = shfl_key(b, 63 - lane);
    a = a > r ? a : r;
    for (int stride = 32; stride > 0; stride >>= 1) a = exchange(a, lane, stride, true);
    return a;
}

// ln(n + s), with the accuracy of log1p where one entry is the maximum
__device__ __forceinline__ float log_total(float n, float s) { return n == 1.f ? log1pf(s) : logf(n + s); }

template <int DT>
__device__ __forceinline__ float logit_at(const void *row, long i)
{
    if constexpr (DT == 2)
        return ((const float *)row)[i];
    else
        return cvt16<DT == 1>(((const uint16_t *)row)[i]);
}

// what a row's sums say: log p of the given token, entropy, statistics for the backward pass; one thread
template <int DT>
__device__ __forceinline__ void write_row(const ScoreArgs &a, int row, const void *z, float m, float n, float s, float q,
                                          float lt)
{
    const bool empty = m == -INFINITY;
    const float total = n + s;
    const float h = empty ? 0.f : lt - LN2 * (q / total);
    if (a.logprob) {
        const int t = a.token[row];
        float lp = 0.f;
        if (t >= 0 && t < a.V) lp = empty ? -INFINITY : (logit_at<DT>(z, t) - m) - lt;
        a.logprob[row] = lp;
    }
    if (a.entropy) a.entropy[row] = h;
    if (a.stats) a.stats[row] = float4_t{empty ? 0.f : m, empty ? 1.f : total, lt, h};
}

// one alternative; key 0: none left.  poison: a NaN or +inf somewhere in the row
__device__ __forceinline__ void write_alternative(const ScoreArgs &a, int row, int j, key_t key, float m, float lt,
                                                  bool poison)
{
    const bool none = key == 0 || poison;
    a.alt_token[(long)row * a.k + j] = none ? -1 : (int32_t)~(uint32_t)key;
    a.alt_logprob[(long)row * a.k + j] =
        poison ? NAN : none ? -INFINITY : (value_of((uint32_t)(key >> 32)) - m) - lt;
}

template <int DT>
__global__ __launch_bounds__(PT) void score_kernel(const ScoreArgs a)
{
    constexpr int E = Piece<DT>::E;
    __shared__ float red[5][PT / 64];                  // of each wave: maximum, smallest group maximum; n, s, q
    __shared__ int count, scan[PT / 64];
    __shared__ key_t cand[PCAP], sorted[PT / 64][64];
    const int T = blockDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = T >> 6;
    const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
    const int whole = a.V / E, rest = a.V - whole * E;                 // whole pieces of the row, entries of its last one
    const int pieces = whole + (rest > 0);
    const int p0 = split * a.seg, p1 = p0 + a.seg < pieces ? p0 + a.seg : pieces;
    const char *z = (const char *)a.z + (long)row * a.stride * (DT == 2 ? 4 : 2);
    if (tid == 0) count = 0;

    Piece<DT> r[PCH];
    float pm[PCH], mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < PCH; ++i) {
        if (p0 + i * T >= p1) break;
        const int p = p0 + tid + i * T;
        if (p < whole && p < p1)
            r[i].w = *(const loose_t *)(z + 16 * (long)p);
        else
            r[i].load_part(z, (long)p * E, p == whole && p < p1 ? rest : 0);
    }
#pragma unroll
    for (int i = 0; i < PCH; ++i) {
        if (p0 + i * T >= p1) break;
        pm[i] = r[i].max();
        mx = fmaxf(mx, pm[i]);
    }
    // the wave's maximum and, for alternatives, the smallest maximum of its groups of `width` lanes: T / width >= k
    float gm = mx;
    {
        int width = 64;
        if (a.k > 0)
            while (width > 1 && T / width < a.k) width >>= 1;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            mx = fmaxf(mx, __shfl_xor(mx, off, WAVE));
            if (a.k > 0) {
                const float o = __shfl_xor(gm, off, WAVE);
                gm = off < width ? fmaxf(gm, o) : fminf(gm, o);
            }
        }
        if (lane == 0) {
            red[0][wave] = mx;
            red[1][wave] = gm;
        }
    }
    __syncthreads();
    float m = red[0][0], tau = red[1][0];
    for (int w = 1; w < waves; ++w) {
        m = fmaxf(m, red[0][w]);
        tau = fminf(tau, red[1][w]);
    }

    // the sums: n entries equal to m, s = sum of exp(z - m) over the others, q = sum of exp(z - m) log2 exp(z - m)
    const float base = m == -INFINITY ? 0.f : m;
    float n = 0.f, s = 0.f, q = 0.f;
    const bool moments = a.entropy || a.stats;
#pragma unroll
    for (int i = 0; i < PCH; ++i) {
        if (p0 + i * T >= p1) break;
        float ps = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = (r[i].val(e) - base) * LOG2E;
            const float w = exp2_hw(x);
            ps += w;
            if (moments) q = fmaf(w, fmaxf(x, NOTHING), q);
        }
        if (pm[i] == m || (a.k > 0 && pm[i] > tau)) {                  // few pieces: the maximum, and candidates
            ps = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float v = r[i].val(e);
                if (v == m)
                    n += 1.f;
                else
                    ps += exp2_hw((v - base) * LOG2E);
                if (a.k > 0 && v > tau) {
                    const int at = atomicAdd(&count, 1);
                    if (at < PCAP) cand[at] = (key_t)order_of(v) << 32 | ~(uint32_t)((p0 + tid + i * T) * E + e);
                }
            }
        }
        s += ps;
    }
    if (m == -INFINITY) n = 0.f;                                       // every entry is masked (a NaN shows in s)
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        n += __shfl_xor(n, off, WAVE);
        s += __shfl_xor(s, off, WAVE);
        q += __shfl_xor(q, off, WAVE);
    }
    if (lane == 0) {
        red[2][wave] = n;
        red[3][wave] = s;
        red[4][wave] = q;
    }
    __syncthreads();
    n = red[2][0], s = red[3][0], q = red[4][0];
    for (int w = 1; w < waves; ++w) {
        n += red[2][w];
        s += red[3][w];
        q += red[4][w];
    }
    const bool poison = !(s < INFINITY) || m == INFINITY;
    const float lt = poison ? NAN : m == -INFINITY ? 0.f : log_total(n, s);
    if (a.splits > 1) {
        if (tid == 0) a.part[(long)row * a.splits + split] = float4_t{m, n, poison ? NAN : s, q};
    } else if (tid == 0) {
        write_row<DT>(a, row, z, poison ? NAN : m, n, s, poison ? NAN : q, lt);
    }
    if (a.k == 0) return;

    int got = poison ? 0 : count;
    uint32_t t = order_of(tau);                                        // entries above t are in the list
    if (got > PCAP) {                                                  // too many: raise t
        uint32_t lo = t, hi = order_of(m);                             // more than PCAP above lo, none above hi
        while (hi - lo > 1) {
            t = lo + (hi - lo) / 2;
            __syncthreads();
            if (tid == 0) count = 0;
            __syncthreads();
            int mine = 0;
#pragma unroll
            for (int i = 0; i < PCH; ++i) {
                if (p0 + i * T >= p1) break;
#pragma unroll
                for (int e = 0; e < E; ++e) mine += order_of(r[i].val(e)) > t;
            }
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) mine += __shfl_xor(mine, off, WAVE);
            if (lane == 0) atomicAdd(&count, mine);
            __syncthreads();
            got = count;
            if (got > PCAP)
                lo = t;
            else if (got < a.k)
                hi = t;
            else
                break;
        }
        if (got > PCAP || got < a.k) t = hi;           // lo and hi met: fewer than k above hi, the others equal it
        __syncthreads();
        if (tid == 0) count = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PCH; ++i) {
            if (p0 + i * T >= p1) break;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t o = order_of(r[i].val(e));
                if (o > t) cand[atomicAdd(&count, 1)] = (key_t)o << 32 | ~(uint32_t)((p0 + tid + i * T) * E + e);
            }
        }
        __syncthreads();
        got = count;
    }
    if (got < a.k && t > ORDER_NINF && !poison) {      // entries equal to t, lowest index first, until there are k
        int have = got;
#pragma unroll
        for (int i = 0; i < PCH; ++i) {
            if (p0 + i * T >= p1 || have >= a.k) break;
            int mine = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) mine += order_of(r[i].val(e)) == t;
            int upto = mine;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int o = __shfl_up(upto, off, WAVE);
                if (lane >= off) upto += o;
            }
            if (lane == 63) scan[wave] = upto;
            __syncthreads();
            int at = have + upto - mine;
            for (int w = 0; w < waves; ++w) {
                at += w < wave ? scan[w] : 0;
                have += scan[w];
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (order_of(r[i].val(e)) == t) {
                    if (at < a.k) cand[at] = (key_t)t << 32 | ~(uint32_t)((p0 + tid + i * T) * E + e);
                    ++at;
                }
            __syncthreads();
        }
        got = have < a.k ? have : a.k;
    }
    // sorted by waves, 64 keys at a time, then joined by the first wave
    const int chunks = (got + 63) / 64;
    key_t best = 0;
    for (int c = wave; c < chunks; c += waves) {
        const int at = c * 64 + lane;
        const key_t v = sort64(at < got ? cand[at] : 0, lane);
        best = best == 0 && c == wave ? v : merge64(best, v, lane);
    }
    if (chunks > 1) {
        sorted[wave][lane] = best;
        __syncthreads();
    }
    if (wave > 0) return;
    for (int w = 1; w < waves && w < chunks; ++w) best = merge64(best, sorted[w][lane], lane);
    if (lane >= a.k) return;
    if (a.splits > 1)
        a.lists[((long)row * a.splits + split) * a.k + lane] = best;
    else
        write_alternative(a, row, lane, best, m, lt, poison);
}

// joins the segments of a row; one wave a row
template <int DT>
__global__ __launch_bounds__(64) void score_join_kernel(const ScoreArgs a)
{
    const int row = blockIdx.x, lane = threadIdx.x;
    const float4_t *part = a.part + (long)row * a.splits;
    float m = -INFINITY;
    bool bad = false;
    for (int i = lane; i < a.splits; i += 64) {
        m = fmaxf(m, part[i][0]);
        bad |= part[i][2] != part[i][2];
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, WAVE));
    const bool poison = __any(bad);
    // a segment's sums, taken from its own maximum to the row's: exp(z - m) = f exp(z - mi), and its n entries join s
    float n = 0.f, s = 0.f, q = 0.f;
    for (int i = lane; i < a.splits; i += 64) {
        const float4_t v = part[i];
        if (v[0] == -INFINITY) continue;
        if (v[0] == m) {
            n += v[1];
            s += v[2];
            q += v[3];
        } else {
            const float x = fmaxf((v[0] - m) * LOG2E, NOTHING), f = exp2_hw(x), total = v[1] + v[2];
            s += f * total;
            q += f * fmaf(x, total, v[3]);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        n += __shfl_xor(n, off, WAVE);
        s += __shfl_xor(s, off, WAVE);
        q += __shfl_xor(q, off, WAVE);
    }
    const float lt = poison ? NAN : m == -INFINITY ? 0.f : log_total(n, s);
    const char *z = (const char *)a.z + (long)row * a.stride * (DT == 2 ? 4 : 2);
    if (lane == 0) write_row<DT>(a, row, z, poison ? NAN : m, n, s, poison ? NAN : q, lt);
    if (a.k == 0) return;
    const key_t *lists = a.lists + (long)row * a.splits * a.k;
    key_t best = lane < a.k ? lists[lane] : 0;
    for (int i = 1; i < a.splits; ++i) best = merge64(best, lane < a.k ? lists[(long)i * a.k + lane] : 0, lane);
    if (lane < a.k) write_alternative(a, row, lane, best, m, lt, poison);
}

struct ScoreGradArgs {
    const void *z;
    void *dz;
    long stride, d_stride;
    const int32_t *token;
    const float4_t *stats;
    const float *d_logprob, *d_entropy;
    int M, V, segs;                  // segments of GT * GCH pieces of a row
};
constexpr int GT = 256, GCH = 4;

template <int DT>
__global__ __launch_bounds__(GT) void score_grad_kernel(const ScoreGradArgs a)
{
    constexpr int E = Piece<DT>::E, SIZE = DT == 2 ? 4 : 2;
    const int row = blockIdx.x / a.segs, seg = blockIdx.x - row * a.segs;
    const int whole = a.V / E, rest = a.V - whole * E;
    const int p0 = seg * GT * GCH + threadIdx.x;
    const char *z = (const char *)a.z + (long)row * a.stride * SIZE;
    char *dz = (char *)a.dz + (long)row * a.d_stride * SIZE;
    const int t = a.token ? a.token[row] : -1;
    const bool given = t >= 0 && t < a.V;
    const float g = given && a.d_logprob ? a.d_logprob[row] : 0.f, h = a.d_entropy ? a.d_entropy[row] : 0.f;
    const bool nothing = g == 0.f && h == 0.f;                         // a row of zeros, whatever its logits
    const float4_t st = a.stats[row];
    const float m = st[0], inv = 1.f / st[1], c = h * (st[3] - st[2]) + g, hl = h * LN2;   // g + h (log p + H) = hl x + c
    Piece<DT> r[GCH];
    if (!nothing) {
#pragma unroll
        for (int i = 0; i < GCH; ++i) {
            const int p = p0 + i * GT;
            if (p < whole)
                r[i].w = *(const loose_t *)(z + 16 * (long)p);
            else
                r[i].load_part(z, (long)p * E, p == whole ? rest : 0);
        }
    }
#pragma unroll
    for (int i = 0; i < GCH; ++i) {
        const int p = p0 + i * GT;
        if (p > whole || (p == whole && rest == 0)) break;
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = (r[i].val(e) - m) * LOG2E;
            o[e] = nothing ? 0.f : -(exp2_hw(x) * inv) * fmaf(hl, fmaxf(x, NOTHING), c);
        }
        if (given && t / E == p) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (t % E == e) o[e] += g;
        }
        u32x4_t w;
        if constexpr (DT == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(o[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e += 2) w[e >> 1] = to16<DT == 1>(o[e]) | (uint32_t)to16<DT == 1>(o[e + 1]) << 16;
        }
        if (p < whole) {
            *(loose_t *)(dz + 16 * (long)p) = w;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < rest) {
                    if constexpr (DT == 2)
                        ((uint32_t *)dz)[(long)p * E + e] = w[e];
                    else
                        ((uint16_t *)dz)[(long)p * E + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
        }
    }
}

inline int pieces_of(int V, int dt) { return (int)(((long)V + (dt == 2 ? 3 : 7)) / (dt == 2 ? 4 : 8)); }

template <int DT>
void launch_score(const ScoreArgs &a, int threads, hipStream_t s)
{
    QLORA_LAUNCH((score_kernel<DT>), dim3((unsigned)(a.M * a.splits)), dim3(threads), 0, s, a);
    if (a.splits > 1) QLORA_LAUNCH((score_join_kernel<DT>), dim3(a.M), dim3(64), 0, s, a);
}

}  // namespace

ScorePlan score_plan(int M, int V, int dt)
{
    const int pieces = pieces_of(V, dt);
    ScorePlan p;
    p.splits = (pieces + PT * PCH - 1) / (PT * PCH);
    p.seg = (pieces + p.splits - 1) / p.splits;
    p.threads = 64;
    while (p.threads < PT && p.threads * 2 < p.seg) p.threads *= 2;
    while (p.threads * PCH < p.seg) p.threads *= 2;
    return p;
}

size_t score_workspace_bytes(int M, int V, int k, int dt)
{
    const ScorePlan p = score_plan(M, V, dt);
    return p.splits == 1 ? 0 : (size_t)M * p.splits * (sizeof(float4_t) + sizeof(key_t) * k);
}

void launch_token_logprobs(const void *logits, long stride, const int32_t *tokens, float *logprob, float *entropy,
                           int32_t *alt_tokens, float *alt_logprobs, int k, float *stats, int M, int V, int dt,
                           void *workspace, hipStream_t s)
{
    const ScorePlan p = score_plan(M, V, dt);
    float4_t *part = (float4_t *)workspace;
    const ScoreArgs a{logits, stride, tokens, logprob, entropy, alt_tokens, alt_logprobs, (float4_t *)stats, M, V, k,
                      p.splits, p.seg, part, (key_t *)(part + (p.splits > 1 ? (size_t)M * p.splits : 0))};
    if (dt == 0)
        launch_score<0>(a, p.threads, s);
    else if (dt == 1)
        launch_score<1>(a, p.threads, s);
    else
        launch_score<2>(a, p.threads, s);
}

void launch_token_logprobs_bwd(const void *logits, long stride, const int32_t *tokens, const float *stats,
                               const float *d_logprob, const float *d_entropy, void *dlogits, long d_stride, int M, int V,
                               int dt, hipStream_t s)
{
    const int segs = (pieces_of(V, dt) + GT * GCH - 1) / (GT * GCH);
    const ScoreGradArgs a{logits, dlogits, stride, d_stride, tokens, (const float4_t *)stats, d_logprob, d_entropy, M, V, segs};
    const dim3 grid((unsigned)((long)M * segs));
    if (dt == 0)
        QLORA_LAUNCH((score_grad_kernel<0>), grid, dim3(GT), 0, s, a);
    else if (dt == 1)
        QLORA_LAUNCH((score_grad_kernel<1>), grid, dim3(GT), 0, s, a);
    else
        QLORA_LAUNCH((score_grad_kernel<2>), grid, dim3(GT), 0, s, a);
}

}  // namespace qlora
