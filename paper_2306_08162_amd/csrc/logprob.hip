// Log probabilities of given tokens, the entropy and the most likely alternatives of each row of logits, and the
// gradient of the first two with respect to the logits.
//
//   m = max z,  S = sum_i exp(z_i - m),   log p_i = (z_i - m) - ln S
//   entropy   H = -sum_i p_i log p_i = ln S + sum_i exp(z_i - m) (m - z_i) / S
//   gradient  of g log p_t + h H:   dz_i = g [i = t] - p_i (g + h (log p_i + H))
//
// The work is bound by HBM: a row is read once (and, backward, once more and its gradient written).  One workgroup takes
// up to 128 KB of a row into registers, so the maximum is known before the first exponential and no sum is ever rescaled;
// longer rows, and rows too few to fill the chip, are cut into segments whose results a second launch joins.  2048 rows of
// 32000 in fp16, 131 MB: 26.3 us or 5.0 TB/s for the log probabilities alone (reading them takes 24), 29 with the entropy, 35 to
// 37 with 20 alternatives besides: an entry costs three instructions, one of them the exponential, and two more with the entropy.
//
// A token that is almost certain has p = 1 / (1 + s) with a tiny s, and S = 1 + s would round it away: the sums keep
// the entries equal to the maximum as a count n apart from the sum s of all others, ln S = log1p(s) where n = 1, and
// log p and H of such a row keep their relative accuracy.  So does the gradient at the token, g (1 - p) = -g expm1(log p).
//
// Alternatives.  Of its lanes' largest entries each of a workgroup's w waves finds (nearly) the ceil(k / w)-th, by bisection
// with ballots; at least k entries are not below tau, the smallest of the w, and on rows in no special order not many more.
// Those above tau are collected in LDS as 64-bit keys (value, lower index first), and a key's place among them is the number
// of larger ones.  Rows that break the rule of thumb (an ordered vocabulary, masks of the type's lowest number) take exact
// detours: the threshold is raised by bisection until the entries above it fit, and entries equal to it are taken in
// order of their index.  Of 2048 x 32000 fp16 with 20 alternatives equal values take 43 us, rising ones 137, falling ones 259.
#include "../../include/qlora.h"
#include "common.hpp"
#include "kernels.hpp"

#include <algorithm>

namespace qlora {

namespace {

constexpr int PCAP = 512;            // keys that LDS holds
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// x log2 of a weight that is zero: far below what exp2 can represent, and finite, so that 0 * x stays 0
constexpr float NOTHING = -1024.f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// max(x, NOTHING) for x <= a little above 0 (see max3 below for why not fmaxf)
__device__ __forceinline__ float nothing_less(float x) { return __builtin_amdgcn_fmed3f(x, NOTHING, 1024.f); }

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

// The maximum that passes over NaN, in one instruction: fmaxf on bits just loaded costs the compiler another one for each
// operand, to quiet a signalling NaN.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

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
            return max3((float)v[0], (float)v[1], (float)v[1]);
        } else if constexpr (DT == 1) {
            return max3(max3(max3(val(0), val(1), val(2)), val(3), val(4)), max3(val(5), val(6), val(7)), val(7));
        } else {
            return max3(max3(val(0), val(1), val(2)), val(3), val(3));
        }
    }
    // -inf weighs nothing and is no alternative
    __device__ __forceinline__ void clear()
    {
        constexpr uint32_t ninf = DT == 2 ? 0xff800000u : DT == 1 ? 0xff80ff80u : 0xfc00fc00u;
        w = u32x4_t{ninf, ninf, ninf, ninf};
    }
    // entries [0, have) of a row's last piece, have < E
    __device__ __forceinline__ void load_part(const void *row, long at, int have)
    {
        clear();
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
            if (e < have) {
                if constexpr (DT == 2) {
                    w[e] = ((const uint32_t *)row)[at + e];
                } else {
                    const uint32_t v = ((const uint16_t *)row)[at + e];
                    w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | v << 16 : (w[e >> 1] & 0xffff0000u) | v;
                }
            }
    }
};

// Lane 63 gathers its wave's values along rows of 16 lanes and from row to row (six steps without LDS), and hands the
// result to all.  KEEP: what a lane without a partner combines with.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float keep, float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(keep), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <typename F>
__device__ __forceinline__ float wave_gather(float v, float keep, F f)
{
    v = f(v, dpp<0x111, 0xf>(keep, v));
    v = f(v, dpp<0x112, 0xf>(keep, v));
    v = f(v, dpp<0x114, 0xf>(keep, v));
    v = f(v, dpp<0x118, 0xf>(keep, v));
    v = f(v, dpp<0x142, 0xa>(keep, v));
    v = f(v, dpp<0x143, 0xc>(keep, v));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_most(float v)
{
    return wave_gather(v, -INFINITY, [](float a, float b) { return max3(a, b, b); });
}
__device__ __forceinline__ float wave_least(float v)
{
    return -wave_gather(-v, -INFINITY, [](float a, float b) { return max3(a, b, b); });
}
__device__ __forceinline__ float wave_total(float v)
{
    return wave_gather(v, 0.f, [](float a, float b) { return a + b; });
}

// the sum over the eight lanes around a lane, all of them active
__device__ __forceinline__ int sum8(int v)
{
    v += __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);            // lane ^ 1
    v += __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);            // lane ^ 2
    return v + __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true);     // lane ^ 7: the other four's sum
}

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
__device__ __forceinline__ void write_row(const ScoreArgs &a, int row, bool given, float zt, float m, float n, float s,
                                          float q, float lt)
{
    const bool empty = m == -INFINITY;
    const float total = n + s;
    const float h = empty ? 0.f : lt - LN2 * (q / total);
    if (a.logprob) a.logprob[row] = !given ? 0.f : empty ? -INFINITY : (zt - m) - lt;
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

// piece i of the registers (a register has no address: i picks among them)
template <int DT, int PCH>
__device__ __forceinline__ Piece<DT> pick(const Piece<DT> *r, int i)
{
    Piece<DT> v = r[0];
#pragma unroll
    for (int j = 1; j < PCH; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v.w[e] = i == j ? r[j].w[e] : v.w[e];
    return v;
}

// MOMENTS: the entropy is asked for, or the statistics that hold it.  At most PT threads with PCH pieces each.
// All of a thread's pieces are requested at once and nothing else is until they are used up: other workgroups of the compute
// unit read meanwhile.  (Stages of four pieces, the next ones on their way, with a maximum of their own: 28.8 us where this takes
// 26.7, for the sums have to be rescaled.)
template <int DT, bool MOMENTS, int PT, int PCH>
__global__ __launch_bounds__(PT) void score_kernel(const ScoreArgs a)
{
    constexpr int E = Piece<DT>::E;
    __shared__ float red[5][PT / 64];                  // of each wave: maximum, bound of its alternatives; n, s, q
    __shared__ float log_s;
    __shared__ int hits, count, scan[PT / 64];
    __shared__ u32x4_t held[PCAP];                     // pieces with an entry above tau, and which they are
    __shared__ int held_at[PCAP];
    __shared__ key_t cand[PCAP];                       // entries above tau
    const int T = blockDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = T >> 6;
    const int row = blockIdx.x, split = blockIdx.y;
    const int whole = a.V / E, rest = a.V - whole * E;                 // whole pieces of the row, entries of its last one
    const int pieces = whole + (rest > 0);
    const int p0 = split * a.seg, p1 = p0 + a.seg < pieces ? p0 + a.seg : pieces;
    const char *z = (const char *)a.z + (long)row * a.stride * (DT == 2 ? 4 : 2);
    const bool last_wave = wave == waves - 1;
    if (tid == 0) hits = count = 0;
    const int token = a.splits == 1 && last_wave && a.logprob ? a.token[row] : -1;

    Piece<DT> r[PCH];
    float pm[PCH], mx = -INFINITY;
    const int full = (p1 < whole ? p1 : whole) - p0;                   // whole pieces of the segment
#pragma unroll
    for (int i = 0; i < PCH; ++i) {
        if (p0 + i * T >= p1) break;
        const char *at = z + 16 * (long)(p0 + i * T);
        if ((i + 1) * T <= full) {
            r[i].w = *(const loose_t *)(at + 16u * (uint32_t)tid);
        } else {
            r[i].clear();
            if (i * T + tid < full) r[i].w = *(const loose_t *)(at + 16u * (uint32_t)tid);
        }
    }
    const bool given = token >= 0 && token < a.V;
    const float zt = given ? logit_at<DT>(z, token) : NAN;             // on its way with the pieces
    if (rest > 0 && p1 == pieces && ((whole - p0) & (T - 1)) == tid) { // the row's last, short piece
        Piece<DT> last;
        last.load_part(z, (long)whole * E, rest);
        const int mine = (whole - p0) / T;
#pragma unroll
        for (int i = 0; i < PCH; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[i].w[e] = mine == i ? last.w[e] : r[i].w[e];
    }
#pragma unroll
    for (int i = 0; i < PCH; ++i) {
        if (p0 + i * T >= p1) break;
        pm[i] = r[i].max();
        mx = max3(mx, pm[i], pm[i]);
    }
    {       // the wave's maximum; for alternatives a bound that `rank` of its lanes' maxima reach
        const float hi = wave_most(mx);
        float bound = hi;
        if (a.k > 0) {
            const int rank = (a.k + waves - 1) / waves;
            // a second largest takes one more reduction (16 x 32000 fp32 with 20: 9.2 -> 8.5 us), further ones as long as the
            // bisection or longer (2048 x 4096 with 5, a third largest: 10.1 -> 10.8)
            if (rank <= 2) {
                if (rank == 2 && __popcll(__ballot(mx >= hi)) < 2) bound = wave_most(mx < hi ? mx : -INFINITY);
            } else {
                const uint32_t mine = order_of(mx);
                uint32_t l = __builtin_amdgcn_readfirstlane(order_of(wave_least(mx))),
                         h = __builtin_amdgcn_readfirstlane(order_of(hi));
                int reach = 64;                                        // so many lanes reach l
                for (int i = 0; i < 12 && reach > rank + rank / 4 && h - l > 1; ++i) {
                    const uint32_t mid = l + (h - l) / 2;
                    const int above = __popcll(__ballot(mine >= mid));
                    if (above >= rank) {
                        l = mid;
                        reach = above;
                    } else {
                        h = mid;
                    }
                }
                bound = value_of(l);
            }
        }
        if (lane == 0) {
            red[0][wave] = hi;
            red[1][wave] = bound;
        }
    }
    __syncthreads();
    const float m = wave_most(lane < waves ? red[0][lane] : -INFINITY);
    const float tau = a.k > 0 ? wave_least(lane < waves ? red[1][lane] : INFINITY) : m;

    // The sums: n entries equal to m, s = sum of w = exp(z - m) over the others, q = sum of w log2 w.  x = z log2 e - base with
    // base = m log2 e rounded is one fused operation on the entry as it lies in the register; the rounding of base is the same
    // factor 2^slip in every w, and is taken off at the end.  Pieces that hold the maximum are left out.
    // Of a maximum so large that its product would leave the range, every other entry is so far away that its weight is zero by
    // any factor.
    const float factor = fabsf(m) < 0x1p126f ? LOG2E : 0.25f;
    const float base = m == -INFINITY ? 0.f : m * factor;
    const float slip = m == -INFINITY ? 0.f : fmaf(m, factor, -base);
    float n = 0.f, s = 0.f, q = 0.f;
    const float low = a.k > 0 ? tau : m;
#pragma unroll
    for (int i = 0; i < PCH; ++i) {
        if (p0 + i * T >= p1) break;
        float x[E], w[E], ps = 0.f, pq = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = fmaf(r[i].val(e), factor, -base);
            w[e] = exp2_hw(x[e]);
            ps += w[e];
            if constexpr (MOMENTS) pq = fmaf(w[e], nothing_less(x[e]), pq);
        }
        if (__any(pm[i] >= low)) {
            if (pm[i] == m) {
                ps = pq = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool top = r[i].val(e) == m;
                    n += top ? 1.f : 0.f;
                    w[e] = top ? 0.f : w[e];
                    ps += w[e];
                    if constexpr (MOMENTS) pq = fmaf(w[e], nothing_less(x[e]), pq);
                }
            }
            if (a.k > 0 && pm[i] > tau) {
                const int at = atomicAdd(&hits, 1);
                if (at < PCAP) {
                    held[at] = r[i].w;
                    held_at[at] = p0 + tid + i * T;
                }
            }
        }
        s += ps;
        if constexpr (MOMENTS) q += pq;
    }
    if (m == -INFINITY) n = 0.f;                                       // every entry is masked (a NaN shows in s)
    n = wave_total(n);
    s = wave_total(s);
    if constexpr (MOMENTS) q = wave_total(q);
    if (lane == 0) {
        red[2][wave] = n;
        red[3][wave] = s;
        red[4][wave] = q;
    }
    __syncthreads();
    n = wave_total(lane < waves ? red[2][lane] : 0.f);
    s = wave_total(lane < waves ? red[3][lane] : 0.f);
    if constexpr (MOMENTS) q = wave_total(lane < waves ? red[4][lane] : 0.f);
    // w = 2^(x - slip): q = sum of w (x - slip).  A slip below -126 belongs to a maximum past 2^30, every other entry 128 or more
    // beneath it: s and q are exact zeros, and stay so by a factor that is finite (a NaN in s stays one by any).
    const float back = exp2_hw(fminf(-slip, 126.f));
    q = (q - slip * s) * back;
    s *= back;
    const bool poison = !(s < INFINITY) || m == INFINITY;
    if (a.splits > 1) {
        if (tid == 0) a.part[(long)row * a.splits + split] = float4_t{m, n, poison ? NAN : s, q};
    } else if (last_wave) {                            // the logarithm: a hundred instructions that one wave is enough for
        const float lt = poison ? NAN : m == -INFINITY ? 0.f : log_total(n, s);
        if (lane == 0) {
            write_row(a, row, given, zt, poison ? NAN : m, n, poison ? NAN : s, poison ? NAN : q, lt);
            log_s = lt;
        }
    }
    if (a.k == 0) return;

    const int pieces_held = poison ? 0 : hits;
    uint32_t t = order_of(tau);                                        // entries above t are to be in the list
    if (pieces_held <= PCAP) {
        for (int j = tid; j < pieces_held * E; j += T) {
            const float v = logit_at<DT>(held, j);
            if (v > tau) {
                const int at = atomicAdd(&count, 1);
                if (at < PCAP) cand[at] = (key_t)order_of(v) << 32 | ~(uint32_t)(held_at[j / E] * E + j % E);
            }
        }
        __syncthreads();
    }
    int got = count;
    if (pieces_held > PCAP || got > PCAP) {                            // too many: raise t
        uint32_t lo = t, hi = order_of(m);                             // more than PCAP or k above lo, none above hi
        got = PCAP + 1;
        while (hi - lo > 1) {
            t = lo + (hi - lo) / 2;
            __syncthreads();
            if (tid == 0) count = 0;
            __syncthreads();
            int mine = 0;
#pragma unroll 1
            for (int i = 0; p0 + i * T < p1; ++i) {
                const Piece<DT> v8 = pick<DT, PCH>(r, i);
#pragma unroll
                for (int e = 0; e < E; ++e) mine += order_of(v8.val(e)) > t;
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
#pragma unroll 1
        for (int i = 0; p0 + i * T < p1; ++i) {
            const Piece<DT> v8 = pick<DT, PCH>(r, i);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t o = order_of(v8.val(e));
                if (o > t) cand[atomicAdd(&count, 1)] = (key_t)o << 32 | ~(uint32_t)((p0 + tid + i * T) * E + e);
            }
        }
        __syncthreads();
        got = count;
    }
    if (got < a.k && t > ORDER_NINF && !poison) {      // entries equal to t, lowest index first, until there are k
        int have = got;
#pragma unroll 1
        for (int i = 0; p0 + i * T < p1 && have < a.k; ++i) {
            const Piece<DT> v8 = pick<DT, PCH>(r, i);
            int mine = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) mine += order_of(v8.val(e)) == t;
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
                if (order_of(v8.val(e)) == t) {
                    if (at < a.k) cand[at] = (key_t)t << 32 | ~(uint32_t)((p0 + tid + i * T) * E + e);
                    ++at;
                }
            __syncthreads();
        }
        got = have < a.k ? have : a.k;
    }
    // a key's place is the number of larger ones, counted by eight lanes; places beyond the last key hold nothing
    const float lt = log_s;                            // (a barrier ago at least; segments have no use for it)
    for (int c = tid >> 3; c < got; c += T >> 3) {
        const key_t mine = cand[c];
        int place = 0;
#pragma unroll 4
        for (int j = tid & 7; j < got; j += 8) place += cand[j] > mine;
        place = sum8(place);
        if ((tid & 7) == 0 && place < a.k) {
            if (a.splits > 1)
                a.lists[((long)row * a.splits + split) * a.k + place] = mine;
            else
                write_alternative(a, row, place, mine, m, lt, poison);
        }
    }
    for (int c = got + tid; c < a.k; c += T) {
        if (a.splits > 1)
            a.lists[((long)row * a.splits + split) * a.k + c] = 0;
        else
            write_alternative(a, row, c, 0, m, lt, poison);
    }
}

// Joins the segments of a row.  Each wave joins the sums for itself.  With alternatives four waves place the lists' keys, JOIN_T
// at a time behind the best so far, of which a k-th bars all smaller ones: of rows in no special order most lists end there.
// (184 lists of 64 alternatives: 82 us for the whole row, 357 without the bar; 777 rows of four lists of 20: 6.0 us a launch
// where one lane per key counted, 7.8.)
constexpr int JOIN_T = 256;
template <int DT>
__global__ __launch_bounds__(JOIN_T) void score_join_kernel(const ScoreArgs a)
{
    __shared__ key_t keys[2][QLORA_MAX_ALTERNATIVES + JOIN_T];         // the best so far, and the next lists' keys
    __shared__ int fresh[JOIN_T / 64];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int token = a.logprob ? a.token[row] : -1;
    const float4_t *part = a.part + (long)row * a.splits;
    float4_t v = {-INFINITY, 0.f, 0.f, 0.f};
    if (lane < a.splits) v = part[lane];
    const key_t *lists = a.lists + (long)row * a.splits * a.k;
    const int all = a.splits * a.k;
    key_t next = tid < all ? lists[tid] : 0;                           // requested with the rest
    const bool given = token >= 0 && token < a.V;
    const float zt = given ? logit_at<DT>((const char *)a.z + (long)row * a.stride * (DT == 2 ? 4 : 2), token) : NAN;
    float m = v[0];
    bool bad = v[2] != v[2];
    for (int i = lane + 64; i < a.splits; i += 64) {
        m = fmaxf(m, part[i][0]);
        bad |= part[i][2] != part[i][2];
    }
    m = wave_most(m);
    const bool poison = __any(bad);
    // a segment's sums, taken from its own maximum to the row's: exp(z - m) = f exp(z - mi), and its n entries join s
    float n = 0.f, s = 0.f, q = 0.f;
    for (int i = lane; i < a.splits; i += 64) {
        if (i >= 64) v = part[i];
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
    n = wave_total(n);
    s = wave_total(s);
    q = wave_total(q);
    const float lt = poison ? NAN : m == -INFINITY ? 0.f : log_total(n, s);
    if (tid == 0) write_row(a, row, given, zt, poison ? NAN : m, n, poison ? NAN : s, poison ? NAN : q, lt);
    if (a.k == 0) return;
    int best = 0, buf = 0;                                             // keys [0, best) are the best so far, in order
    for (int at = 0; at < all; at += JOIN_T) {
        // key 0 is a place that a short list left open; keys behind the k-th best so far are passed over
        const key_t bar = best == a.k ? keys[buf][best - 1] : 0;
        const bool good = next > bar;
        const uint64_t who = __ballot(good);
        if (lane == 0) fresh[tid >> 6] = __popcll(who);
        __syncthreads();
        int have = best, mine_at = best;
        for (int w = 0; w < JOIN_T / 64; ++w) {
            mine_at += w < tid >> 6 ? fresh[w] : 0;
            have += fresh[w];
        }
        mine_at += __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
        if (good) keys[buf][mine_at] = next;
        next = at + JOIN_T + tid < all ? lists[at + JOIN_T + tid] : 0;
        __syncthreads();
        if (have == best) continue;
        // a key's place is the number of larger ones, counted by eight lanes
        for (int c = tid >> 3; c < have; c += JOIN_T >> 3) {
            const key_t mine = keys[buf][c];
            int place = 0;
#pragma unroll 4
            for (int j = tid & 7; j < have; j += 8) place += keys[buf][j] > mine;
            place = sum8(place);
            if ((tid & 7) == 0 && place < a.k) keys[buf ^ 1][place] = mine;
        }
        __syncthreads();
        best = have < a.k ? have : a.k;
        buf ^= 1;
    }
    if (tid < a.k) write_alternative(a, row, tid, tid < best ? keys[buf][tid] : 0, m, lt, poison);
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

// Elementwise, at the rate of a large copy (2048 x 32000 fp16: 45 us, 5.8 TB/s; 41 right behind the forward pass).  The gradient is stored past the caches: it
// would drive out the logits that the forward pass has just brought there (both passes together 82 us, 69 with the hint); a
// reader that follows at once finds the whole chain as fast or faster (1 to 131 MB of gradient: 0.88 to 1.01 times).
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
    const float m = st[0], inv = 1.f / st[1], hl = h * LN2;
    const float ch = h * (st[3] - st[2]), c = ch + g;                  // h (log p + H) = hl x + ch
    Piece<DT> r[GCH];
    if (!nothing) {
#pragma unroll
        for (int i = 0; i < GCH; ++i) {
            const int p = p0 + i * GT;
            r[i].clear();
            if (p < whole)
                r[i].w = __builtin_nontemporal_load((const loose_t *)(z + 16 * (long)p));
            else if (p == whole && rest > 0)
                r[i].load_part(z, (long)p * E, rest);
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
            float zt = r[i].val(0), o_t = o[0];
#pragma unroll
            for (int e = 1; e < E; ++e) {
                zt = t % E == e ? r[i].val(e) : zt;
                o_t = t % E == e ? o[e] : o_t;
            }
            const float x = (zt - m) * LOG2E, p_t = exp2_hw(x) * inv;
            // g (1 - p): as a difference while that rounds once, by log p where the difference would lose digits
            if (nothing || p_t < 0.5f)
                o_t += g;
            else
                o_t = -g * expm1f((zt - m) - st[2]) - p_t * fmaf(hl, fmaxf(x, NOTHING), ch);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = t % E == e ? o_t : o[e];
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
            __builtin_nontemporal_store(w, (loose_t *)(dz + 16 * (long)p));
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

// Many rows: 256 threads with 64 KB of a row, four workgroups on a compute unit.  2048 x 32000 fp16: 31 us when first built that
// way, 33 with 512 threads and half the pieces, 57 with 1024 and a quarter, 36 with twice the pieces and 128 or 256 threads, whose
// waves are too few.  Rows of 64 to 128 KB: 512 threads, which spares the second launch (1024 x 32000 fp32 26.3 us, 29.5 as two
// segments).  Longer ones in segments of at most 64 KB: 777 x 128259 bf16 with 20 alternatives takes 55.7 us, with 128 KB 61.8,
// with 45 to 22 KB 63 to 72, for each segment has alternatives of its own (without any 42 to 46 us, 51 with 128 KB).
// Few rows (no more than compute units): each has one to itself, and 1024 threads get through it sooner.
constexpr int MANY_PT = 512, MANY_PCH = 16, FEW_PT = 1024, FEW_PCH = 8, SEGMENT = 4096;

inline int pieces_of(int V, int dt) { return (int)(((long)V + (dt == 2 ? 3 : 7)) / (dt == 2 ? 4 : 8)); }

template <int DT>
void launch_score(const ScoreArgs &a, const ScorePlan &p, hipStream_t s)
{
    const dim3 grid(a.M, a.splits), block(p.threads);
    const bool moments = a.entropy || a.stats;
    if (p.threads * FEW_PCH >= p.seg) {
        if (moments)
            QLORA_LAUNCH((score_kernel<DT, true, FEW_PT, FEW_PCH>), grid, block, 0, s, a);
        else
            QLORA_LAUNCH((score_kernel<DT, false, FEW_PT, FEW_PCH>), grid, block, 0, s, a);
    } else {
        if (moments)
            QLORA_LAUNCH((score_kernel<DT, true, MANY_PT, MANY_PCH>), grid, block, 0, s, a);
        else
            QLORA_LAUNCH((score_kernel<DT, false, MANY_PT, MANY_PCH>), grid, block, 0, s, a);
    }
    if (a.splits > 1) QLORA_LAUNCH((score_join_kernel<DT>), dim3(a.M), dim3(a.k > 0 ? JOIN_T : WAVE), 0, s, a);
}

}  // namespace

ScorePlan score_plan(int M, int V, int dt)
{
    const int pieces = pieces_of(V, dt);
    ScorePlan p;
    p.splits = pieces <= MANY_PT * MANY_PCH ? 1 : (pieces + SEGMENT - 1) / SEGMENT;
    const bool many = (long)M * p.splits > 256;
    // one workgroup a row as long as one can hold it; else short segments on as many compute units as there are (8 x 128256 bf16:
    // 11.5 us, 14.1 with as few segments as hold it)
    if (!many) {
        p.splits = (pieces + FEW_PT * FEW_PCH - 1) / (FEW_PT * FEW_PCH);
        const int spread = std::min((pieces + 2047) / 2048, 512 / M);
        if (p.splits > 1) p.splits = std::max(p.splits, spread);
    }
    p.seg = (pieces + p.splits - 1) / p.splits;
    p.threads = 64;
    // of many short rows what a wave does once a row weighs more than its pieces: few waves, as long as the chip has sixteen a unit
    // (2048 x 4096 fp16: 7.6 us, 9.5 with a wave for every 64 pieces)
    if (many) {
        while (p.threads * MANY_PCH < p.seg) p.threads *= 2;
        while (p.threads < 256 && p.threads * 2 < p.seg && (long)M * p.splits * p.threads < 256 * 1024) p.threads *= 2;
    } else {
        while (p.threads < FEW_PT && p.threads * 2 < p.seg) p.threads *= 2;
    }
    return p;
}

size_t score_workspace_bytes(int M, int V, int k, int dt)
{
    const ScorePlan p = score_plan(M, V, dt);
    return p.splits == 1 ? 0 : (size_t)M * p.splits * (sizeof(float4_t) + sizeof(key_t) * k);
}

size_t score_workspace_bound(int M, int V, int k, int dt)
{
    if (score_plan(M, V, dt).splits == 1) return 0;                    // which follows from V alone
    const size_t pieces = pieces_of(V, dt);
    // of many rows each has ceil(pieces / SEGMENT) segments, of few no more than that or the spread of score_plan
    const size_t many = M * ((pieces + SEGMENT - 1) / SEGMENT), few = std::min<size_t>(M * ((pieces + 2047) / 2048), 512);
    return std::max(many, few) * (sizeof(float4_t) + sizeof(key_t) * k);
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
        launch_score<0>(a, p, s);
    else if (dt == 1)
        launch_score<1>(a, p, s);
    else
        launch_score<2>(a, p, s);
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
