// verify.cu -- which drafted tokens the target's probabilities keep, and the
// token that follows them (mtsim_ops.h).
#include "tensor.cuh"

#include <cooperative_groups.h>

namespace mtop {
namespace {

namespace cg = cooperative_groups;

// Two kernels.  k_rows takes all rows of logits in chunks, a block a chunk, and leaves the chunk's largest logit
// and the sum of its weights.  k_draw, a cluster of blocks a request, joins these, decides how many tokens are
// accepted, goes once more over the one row (or the two) that the next token is drawn from, and the
// warp whose stretch holds the point looks for it.
// 64 requests, 4 rows of 131,075 bfloat16 logits and 3 of the draft (117 MB) take 49 us: the rows 25, bound by instructions (11 a
// logit; 62 registers and two blocks a multiprocessor 33; three leave 40 registers, and the bfloat16 kernel has 72 bytes on its stack besides), the draw 21, bound by waiting for its loads.
//
// Nothing is in 64-bit floating point, which runs at a sixtieth of the rate here (with it these two kernels took 165 us for that, 58 of
// them a division by every thread).  Sums of single threads and warps are 32-bit floats, whose errors are independent and average out; sums
// of those are pairs of floats, and the masses that the draw goes by are whole numbers of 2^-50, which add up the same in any order.
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBatch = 4;            // vectors that a thread has on their way
constexpr int kMostCluster = 8;
typedef unsigned long long u64;

// log2(e) / t in two floats: (l - m) * (hi + lo) is the binary logarithm of a weight.  (Not zero for an infinite t:
// -infinity times it is -infinity.)
struct Rate {
    float hi, lo;
    bool greedy;
    // (A 32-bit division and its rest.)
    __device__ __forceinline__ explicit Rate(float t) {
        greedy = !(t > 0.f);
        const float q = 1.44269502f / (greedy ? 1.f : t), rest = fmaf(-q, t, 1.44269502f) + 1.92596303e-8f, more = rest / t;
        hi = fminf(fmaxf(q, 1e-36f), 3e38f), lo = hi == q && fabsf(more) < q * 1e-6f ? more : 0.f;
    }
};

// Two floats in a register pair, so that what is the same for all logits is put into one once.
__device__ __forceinline__ u64 pair_of(float x, float y) {
    u64 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void parts_of(u64 r, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ u64 pair_add(u64 x, u64 y) {
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(y));
    return x;
}
__device__ __forceinline__ u64 pair_mul(u64 x, u64 y) {
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(y));
    return x;
}
__device__ __forceinline__ u64 pair_fma(u64 x, u64 y, u64 z) {
    asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(x) : "l"(y), "l"(z));
    return x;
}

// A chunk, or a whole row: its largest logit, the sum (and what it was rounded by) of the weights 2^(rate (l - top)), and
// the lowest index of the largest (greedy requests: all of the weight).
struct Stat {
    float top, sum, rest;
    int first;
    __device__ __forceinline__ void add(float x) {
        const float s = __fadd_rn(sum, x), b = __fsub_rn(s, sum);
        rest += __fadd_rn(__fsub_rn(sum, __fsub_rn(s, b)), __fsub_rn(x, b));
        sum = s;
    }
};

// A weight to about 2^-22 of itself: the exponent's rounding (2^-24 of up to
// 126) is kept apart and multiplied in.
template <typename T> __device__ __forceinline__ float weight_of(float l, int v, float top, int first, const Rate &c) {
    if (c.greedy) return v == first ? 1.f : 0.f;
    if (!(l > -INFINITY)) return 0.f;  // (or NaN)
    if (top == INFINITY) return l == INFINITY ? 1.f : 0.f;
    const float d = __fsub_rn(l, top);
    float off = 0.f;  // d + off = l - top (16-bit numbers: d is exact, or so far below 0 that it does not matter)
    if (sizeof(T) == 4) {
        const float b = __fsub_rn(d, l);
        off = __fsub_rn(__fsub_rn(l, __fsub_rn(d, b)), __fadd_rn(top, b));
    }
    const float y = __fmul_rn(d, c.hi);
    if (!(y > -126.f)) return 0.f;
    const float e = fmaf(d, c.hi, -y) + fmaf(d, c.lo, off * c.hi), p = exp2_fast(y);
    return fmaf(p, e * 0.6931471805599453f, p);
}

// The weights of a vector's logits, to the same accuracy, where the row's largest is a number.
template <typename T, int N> __device__ __forceinline__ void weights_of(float *l, int v, float top, int first, const Rate &c) {
    if (c.greedy || !(fabsf(top) < INFINITY) || sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < N; ++e) l[e] = weight_of<T>(l[e], v + e, top, first, c);
        return;
    }
    const u64 less = pair_of(-top, -top), hi = pair_of(c.hi, c.hi), lo = pair_of(c.lo, c.lo), minus = pair_of(-1.f, -1.f),
              ln2 = pair_of(0.6931471805599453f, 0.6931471805599453f);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        const u64 d = pair_add(pair_of(l[e], l[e + 1]), less), y = pair_mul(d, hi), off = pair_fma(d, lo, pair_fma(d, hi, pair_mul(y, minus)));
        float y0, y1;
        parts_of(y, y0, y1);
        const u64 p = pair_of(exp2_fast(y0), exp2_fast(y1));
        parts_of(pair_fma(p, pair_mul(off, ln2), p), l[e], l[e + 1]);
        l[e] = y0 > -126.f ? l[e] : 0.f, l[e + 1] = y1 > -126.f ? l[e + 1] : 0.f;
    }
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
__device__ __forceinline__ int warp_min(int v) { return __reduce_min_sync(~0u, v); }

// ------------------------------------------------------------- rows -------
// The 16 bytes at position p of a row whose first logit is `skip` elements after a 16-byte boundary, from which positions
// count (p < vocab + skip: one of them is the row's), as 32-bit numbers; what is not the row's as -infinity.
template <typename T> __device__ __forceinline__ void logits_of(const Vec<T> &x, int p, int skip, int vocab, float *f) {
    constexpr int N = Vec<T>::N;
    x.to(f);
    if (p < skip || p + N > vocab + skip) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (p + e < skip || p + e >= vocab + skip) f[e] = -INFINITY;
    }
}

// A vector of logits as they are held: the largest (NaN left out), and 32-bit pairs of those not below `low`.
template <typename T> struct Held;
template <> struct Held<__nv_bfloat16> {
    static constexpr float low = -1.00000000e+30f;
    __device__ static float largest(const uint4 &x) {
        __nv_bfloat162 m = __hmax2(__hmax2(*(const __nv_bfloat162 *)&x.x, *(const __nv_bfloat162 *)&x.y), __hmax2(*(const __nv_bfloat162 *)&x.z, *(const __nv_bfloat162 *)&x.w));
        const uint32_t w = *(const uint32_t *)&m;
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    __device__ static u64 pair(const uint4 &x, int i) {
        const __nv_bfloat162 m = __hmax2(*(const __nv_bfloat162 *)(&x.x + i), __float2bfloat162_rn(low));
        const uint32_t w = *(const uint32_t *)&m;
        return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
};
template <> struct Held<__half> {
    static constexpr float low = -65504.f;
    __device__ static float largest(const uint4 &x) {
        const __half2 m = __hmax2(__hmax2(*(const __half2 *)&x.x, *(const __half2 *)&x.y), __hmax2(*(const __half2 *)&x.z, *(const __half2 *)&x.w));
        const float2 f = __half22float2(m);
        return fmaxf(f.x, f.y);
    }
    __device__ static u64 pair(const uint4 &x, int i) {
        const float2 f = __half22float2(__hmax2(*(const __half2 *)(&x.x + i), __float2half2_rn(low)));
        return pair_of(f.x, f.y);
    }
};
template <> struct Held<float> {
    static constexpr float low = -1.00000000e+30f;
    __device__ static float largest(const uint4 &x) {
        return fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w)));
    }
    __device__ static u64 pair(const uint4 &x, int i) {
        const uint32_t *w = &x.x + 2 * i;
        return pair_of(fmaxf(__uint_as_float(w[0]), low), fmaxf(__uint_as_float(w[1]), low));
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 3) k_rows(const __grid_constant__ sim_op_verify_t a, Stat *stats, int rows, int chunks, int chunk_len) {
    constexpr int N = Vec<T>::N;
    __shared__ float tops[kWarps], sums[kWarps];
    __shared__ int firsts[kWarps];
    let_next_start();
    after_previous();
    const uint32_t row = blockIdx.x / (uint32_t)chunks, in = row / (uint32_t)rows;
    const int64_t b = in;
    const int chunk = (int)(blockIdx.x - row * chunks), k = (int)(row - in * rows), lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int drafted = a.drafted ? min(max(a.drafted[b], 0), a.drafts) : a.drafts;
    if (k <= a.drafts ? k > drafted : k - a.drafts - 1 >= drafted) return;  // of a token that is not there
    const T *from = k <= a.drafts ? (const T *)a.target + b * a.target_request + k * a.target_row
                                  : (const T *)a.draft + b * a.draft_request + (k - a.drafts - 1) * a.draft_row;
    const Rate c(a.temperature ? a.temperature[b] : 1.f);
    const int skip = (int)(((uintptr_t)from & 15) / sizeof(T)), begin = chunk * chunk_len, end = min(begin + chunk_len, a.vocab + skip);
    const Vec<T> *x = (const Vec<T> *)(from - skip);
    float top = -INFINITY, sum = 0.f;
    int first = 0x7FFFFFFF;
    // Without a branch for a logit's kind: -infinity and NaN count as the lowest number `low`, whose weight is 0 under a
    // logit far above it, and the largest is taken anew with every vector.  Threads that find nothing from which a
    // weight at `low` would be 0 (2^-150: of float16 rows, whose lowest number is an ordinary one), or +infinity, look again below.
    const bool plain = !c.greedy && c.hi < 1e6f && c.hi > 0.01f;
    if (plain) {
        const u64 hi = pair_of(c.hi, c.hi), lo = pair_of(c.lo, c.lo);
        float high = Held<T>::low;
        for (int p0 = begin + threadIdx.x * N; p0 < end; p0 += kBatch * kThreads * N) {
            uint4 v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (p0 + i * kThreads * N < end) v[i] = *(const uint4 *)(x + p0 / N + i * kThreads);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int p = p0 + i * kThreads * N;
                if (p >= end) break;
                if (p < skip || p + N > a.vocab + skip) {
                    T *t = (T *)&v[i];
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (p + e < skip || p + e >= a.vocab + skip) t[e] = elem<T>::from(-INFINITY);
                }
                const float most = Held<T>::largest(v[i]), now = fmaxf(high, most);
                top = fmaxf(top, most);
                sum *= exp2_fast((high - now) * c.hi);
                high = now;
                const u64 less = pair_of(-now, -now);
                u64 part = 0;
#pragma unroll
                for (int e = 0; e < N / 2; ++e) {
                    const u64 d = pair_add(Held<T>::pair(v[i], e), less);
                    float y0, y1;
                    parts_of(pair_fma(d, lo, pair_mul(d, hi)), y0, y1);
                    part = pair_add(part, pair_of(exp2_fast(y0), exp2_fast(y1)));
                }
                float s0, s1;
                parts_of(part, s0, s1);
                sum += s0 + s1;
            }
        }
        if (top == -INFINITY) sum = 0.f;
    }
    // one by one
    const bool again = plain && (top == INFINITY || (top > -INFINITY && (top - Held<T>::low) * c.hi < 150.f));
    if (again) top = -INFINITY, sum = 0.f;
    if (!plain || again) for (int p0 = begin + threadIdx.x * N; p0 < end; p0 += kBatch * kThreads * N) {
        Vec<T> v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (p0 + i * kThreads * N < end) v[i] = x[p0 / N + i * kThreads];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int p = p0 + i * kThreads * N;
            if (p >= end) break;
            float f[N];
            logits_of(v[i], p, skip, a.vocab, f);
            float most = f[0];
#pragma unroll
            for (int e = 1; e < N; ++e) most = fmaxf(most, f[e]);
            if (c.greedy) {
                if (most > top) {
                    top = most;
#pragma unroll
                    for (int e = N - 1; e >= 0; --e)
                        if (f[e] == most) first = p + e - skip;
                }
                continue;
            }
            if (most > top) {
                sum *= exp2_fast((top - most) * c.hi);
                top = most;
                if (top == INFINITY) sum = 0.f;  // from here on only such count
            }
            if (top == INFINITY) {
#pragma unroll
                for (int e = 0; e < N; ++e) sum += f[e] == INFINITY;
            } else if (top > -INFINITY) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = f[e] - top;
                    sum += exp2_fast(fmaxf(fmaf(d, c.lo, d * c.hi), -200.f));  // (of -infinity or NaN: NaN, and so nothing)
                }
            }
        }
    }
    const float high = warp_max(top);
    float s = top == -INFINITY ? 0.f : high == INFINITY ? (top == INFINITY ? sum : 0.f) : sum * exp2_fast((top - high) * c.hi);
    s = warp_sum(s);
    first = warp_min(top == high ? first : 0x7FFFFFFF);
    if (lane == 0) tops[warp] = high, sums[warp] = s, firsts[warp] = first;
    __syncthreads();
    if (warp == 0) {
        const float t = lane < kWarps ? tops[lane] : -INFINITY, all = warp_max(t);
        const int f = warp_min(lane < kWarps && t == all ? firsts[lane] : 0x7FFFFFFF);
        Stat r = {all, lane < kWarps && t > -INFINITY ? (t == all ? sums[lane] : sums[lane] * exp2_fast((t - all) * c.hi)) : 0.f, 0.f, f};
#pragma unroll
        for (int o = kWarps / 2; o; o >>= 1) {
            const float s2 = __shfl_xor_sync(~0u, r.sum, o), r2 = __shfl_xor_sync(~0u, r.rest, o);
            r.add(s2), r.rest += r2;
        }
        if (lane == 0) stats[(int64_t)row * chunks + chunk] = r;
    }
}

// ------------------------------------------------------------- draw -------
// Logits v .. v + N - 1 of a row that begins anywhere (v < vocab, the first may lie before the row), as they lie in one or two vectors of 16 bytes.
template <typename T> __device__ __forceinline__ void logits_at(const T *row, int v, int vocab, float *f) {
    constexpr int N = Vec<T>::N;
    const uintptr_t at = (uintptr_t)(row + v);
    const int shift = (int)(at & 15);
    const uint4 *from = (const uint4 *)(at - shift);
    Vec<T> x;
    uint4 y = v + (16 - shift) / (int)sizeof(T) > 0 ? from[0] : make_uint4(0, 0, 0, 0);  // (each is read where it holds an element of the row)
    if (shift) {
        const uint4 hi = v + (16 - shift) / (int)sizeof(T) < vocab ? from[1] : make_uint4(0, 0, 0, 0);
        uint32_t w[8] = {y.x, y.y, y.z, y.w, hi.x, hi.y, hi.z, hi.w};
        if (shift & 8) {
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
        }
        if (shift & 4) {
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
        }
        const uint32_t by = shift & 2 ? 0x5432 : 0x3210;
        y = make_uint4(__byte_perm(w[0], w[1], by), __byte_perm(w[1], w[2], by), __byte_perm(w[2], w[3], by), __byte_perm(w[3], w[4], by));
    }
    *(uint4 *)&x = y;
    x.to(f);
    if (v < 0 || v + N > vocab) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (v + e < 0 || v + e >= vocab) f[e] = -INFINITY;
    }
}

// A weight that is at most 1 in whole numbers of 2^-50.
__device__ __forceinline__ u64 units_of(float w) { return __float2ull_rz(w * 0x1p50f); }
// floor(x * f) for 0 <= f < 1 (else 0 or the largest below x) and x below 2^63.
__device__ __forceinline__ u64 share_of(u64 x, float f) {
    if (!(f > 0.f)) return 0;
    if (f >= 1.f) return x ? x - 1 : 0;
    const uint32_t b = __float_as_uint(f), e = b >> 23, m = (b & 0x7FFFFF) | (e ? 0x800000 : 0);
    const int shift = 150 - (e ? e : 1);  // f = m / 2^shift, shift >= 24
    const u64 lo = x * m, hi = __umul64hi(x, m);
    return shift < 64 ? hi << (64 - shift) | lo >> shift : shift < 128 ? hi >> (shift - 64) : 0;
}
// (Masses are shares of one row's, so that all together are less than 2^51: their upper parts fit 32 bits.)
__device__ __forceinline__ u64 warp_total(u64 v) {
    return ((u64)__reduce_add_sync(~0u, (unsigned)(v >> 25)) << 25) + __reduce_add_sync(~0u, (unsigned)v & 0x1FFFFFF);
}
__device__ __forceinline__ u64 warp_up_to(u64 v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 u = __shfl_up_sync(~0u, v, o);
        if ((threadIdx.x & 31) >= o) v += u;
    }
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) k_draw(const __grid_constant__ sim_op_verify_t a, const Stat *stats, int rows, int chunks, int stretch) {
    constexpr int N = Vec<T>::N, kParts = kMostCluster * kWarps, kSteps = 16;  // steps whose masses are kept
    __shared__ Stat row_stat[2 * SIM_OP_MAX_DRAFTS + 1];
    __shared__ bool passed[SIM_OP_MAX_DRAFTS];
    __shared__ u64 mass[2][kWarps], ahead_of[kParts], whole;  // mass: of the block's warps' stretches
    __shared__ u64 step_mass[kWarps][kSteps];
    __shared__ int found;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t b = blockIdx.x / (uint32_t)blocks;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    let_next_start();
    after_previous();
    const int drafted = a.drafted ? min(max(a.drafted[b], 0), a.drafts) : a.drafts;
    const Rate c(a.temperature ? a.temperature[b] : 1.f);
    const T *target = (const T *)a.target + b * a.target_request, *draft = a.draft ? (const T *)a.draft + b * a.draft_request : nullptr;
    const int64_t *tokens = a.tokens + b * a.drafts;
    const float *uniform = a.uniform + b * (a.drafts + 1);
    // the rows' chunks, a row a warp
    for (int k = warp; k < rows; k += kWarps) {
        if (k <= a.drafts ? k > drafted : k - a.drafts - 1 >= drafted) continue;
        const Stat *s = stats + (b * rows + k) * chunks;
        Stat r = {-INFINITY, 0.f, 0.f, 0x7FFFFFFF};
        for (int i0 = 0; i0 < chunks; i0 += 32) {  // (one round for up to 32 chunks)
            const Stat x = i0 + lane < chunks ? s[i0 + lane] : Stat{-INFINITY, 0.f, 0.f, 0x7FFFFFFF};
            const float top = fmaxf(r.top, warp_max(x.top));
            const int first = warp_min(x.top == top ? x.first : 0x7FFFFFFF);
            const float by = r.top == top ? 1.f : r.top > -INFINITY && top < INFINITY ? exp2_fast((r.top - top) * c.hi) : 0.f;
            r.sum *= by, r.rest *= by;
            if (top > r.top) r.first = first;
            r.top = top;
            const float own = x.top == top ? 1.f : x.top > -INFINITY && top < INFINITY ? exp2_fast((x.top - top) * c.hi) : 0.f;
            Stat t = {top, x.sum * own, x.rest * own, 0};
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const float s2 = __shfl_xor_sync(~0u, t.sum, o), r2 = __shfl_xor_sync(~0u, t.rest, o);
                t.add(s2), t.rest += r2;
            }
            r.add(t.sum), r.rest += t.rest;
        }
        r.sum = c.greedy ? (float)(r.top > -INFINITY) : r.top > -INFINITY ? r.sum + r.rest : 0.f;
        if (lane == 0) row_stat[k] = r;
    }
    __syncthreads();
    auto chance = [&](float l, int v, const Stat &p) { return p.sum > 0.f ? weight_of<T>(l, v, p.top, p.first, c) / p.sum : 0.f; };
    auto log_p = [&](float l, int v, const Stat &p) {
        if (!(weight_of<T>(l, v, p.top, p.first, c) > 0.f)) return -INFINITY;
        if (c.greedy) return 0.f;
        const float d = l - p.top;
        return (p.top == INFINITY ? 0.f : fmaf(d, c.hi, d * c.lo) * 0.6931471805599453f) - logf(p.sum);
    };
    // every drafted token's test, a token a thread
    if (threadIdx.x < drafted) {
        const int i = threadIdx.x;
        const int64_t x = tokens[i];
        const bool real = x >= 0 && x < a.vocab;
        const float px = real ? chance(elem<T>::to(target[i * a.target_row + x]), (int)x, row_stat[i]) : 0.f;
        const float qx = !real ? 0.f : draft ? chance(elem<T>::to(draft[i * a.draft_row + x]), (int)x, row_stat[a.drafts + 1 + i]) : 1.f;
        passed[i] = uniform[i] * qx < px;
    }
    __syncthreads();
    int at = 0;
    while (at < drafted && passed[at]) ++at;
    // the row that is drawn from, a stretch a warp
    bool refused = at < drafted;
    const Stat p = row_stat[at], q = refused && draft ? row_stat[a.drafts + 1 + at] : Stat{0.f, 0.f, 0.f, 0};
    const T *lp = target + at * a.target_row, *lq = refused && draft ? draft + at * a.draft_row : nullptr;
    const int64_t x = refused ? tokens[at] : -1;
    // Two rows' sums that are no further apart than 2^-20 are taken as one: that is what rounding can make of equal rows whose
    // places in a vector differ and which are summed in other groups (2^-21.3 at most in rows of 1,023 to 1,000,003 logits
    // of many kinds), and what it leaves of p - q must not be drawn from.
    const float by_p = p.sum > 0.f ? 1.f / p.sum : 0.f,
                by_q = fabsf(p.sum - q.sum) <= 0x1p-20f * p.sum ? by_p : q.sum > 0.f ? 1.f / q.sum : 0.f;
    const int skip = (int)(((uintptr_t)lp & 15) / sizeof(T)), end_at = a.vocab + skip;  // positions count from a boundary
    auto weights = [&](int pos, float *w) {
        const int v = pos - skip;
        logits_of(*(const Vec<T> *)(lp + v), pos, skip, a.vocab, w);
        weights_of<T, N>(w, v, p.top, p.first, c);
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = __fmul_rn(w[e], by_p);
        if (!refused) return;
        if (lq) {
            float g[N];
            logits_at(lq, v, a.vocab, g);
            weights_of<T, N>(g, v, q.top, q.first, c);
            // (two roundings and not one fused step: equal probabilities leave nothing)
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = fmaxf(__fsub_rn(w[e], __fmul_rn(g[e], by_q)), 0.f);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (v + e == x) w[e] = fmaxf(__fsub_rn(w[e], 1.f), 0.f);
        }
    };
    auto units = [&](const float *w) {
        u64 s = pair_of(w[0], w[1]);
#pragma unroll
        for (int e = 2; e < N; e += 2) s = pair_add(s, pair_of(w[e], w[e + 1]));
        float s0, s1;
        parts_of(s, s0, s1);
        return units_of(s0 + s1);
    };
    const int part = rank * kWarps + warp, begin = part * stretch, end = min(begin + stretch, end_at);
    int chosen = -1;  // the part with the point
    u64 want = 0;
    for (int round = 0; round < 2; ++round) {
        u64 sum = 0;
        for (int p0 = begin, k = 0; p0 < end; p0 += 32 * N, ++k) {
            const int pos = p0 + lane * N;
            float w[N];
            u64 own = 0;
            if (pos < end) weights(pos, w), own = units(w);
            if (k < kSteps) {
                own = warp_total(own);
                if (lane == 0) step_mass[warp][k] = own;
                sum += lane == 0 ? own : 0;
            } else {
                sum += own;
            }
        }
        sum = warp_total(sum);
        if (lane == 0) mass[round][warp] = sum;
        if (blocks > 1) cluster.sync();
        else __syncthreads();
        const int parts = blocks * kWarps;
        if (warp == 0) {
            // the masses ahead of every part, four parts a lane
            u64 m[kParts / 32], all = 0;
#pragma unroll
            for (int k = 0; k < kParts / 32; ++k) {
                const int i = lane * (kParts / 32) + k;
                m[k] = i >= parts ? 0 : blocks > 1 ? cluster.map_shared_rank(&mass[round][0], i / kWarps)[i % kWarps] : mass[round][i];
                all += m[k];
            }
            const u64 up_to = warp_up_to(all), total = __shfl_sync(~0u, up_to, 31), point = share_of(total, uniform[a.drafts]);
            u64 run = up_to - all;
            int here = 0x7FFFFFFF;
#pragma unroll
            for (int k = 0; k < kParts / 32; ++k) {
                const int i = lane * (kParts / 32) + k;
                if (i < parts) ahead_of[i] = run;
                run += m[k];
                if (run > point && here == 0x7FFFFFFF) here = i;
            }
            here = warp_min(here);
            if (lane == 0) whole = total, found = total ? here : -1;
        }
        __syncthreads();
        chosen = found, want = share_of(whole, uniform[a.drafts]);
        if (chosen >= 0 || !refused) break;
        refused = false;  // nothing is left: from p itself
        __syncthreads();
    }
    int64_t *out = a.out + b * (a.drafts + 1);
    float *logprob = a.logprob ? a.logprob + b * (a.drafts + 1) : nullptr;
    auto drawn = [&](int token) {
        out[at] = token;
        if (logprob) logprob[at] = token < 0 ? -INFINITY : log_p(elem<T>::to(lp[token]), token, p);
        a.count[b] = at + 1;
    };
    if (chosen == part) {
        u64 before = ahead_of[part];
        int token = -1, p0 = begin;
        for (int k = 0; k < kSteps && p0 < end && before + step_mass[warp][k] <= want; ++k) before += step_mass[warp][k], p0 += 32 * N;
        for (; p0 < end && token < 0; p0 += 32 * N) {
            const int pos = p0 + lane * N;
            float w[N];
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = 0.f;
            if (pos < end) weights(pos, w);
            const u64 own = units(w), up_to = warp_up_to(own);
            const unsigned above = __ballot_sync(~0u, before + up_to > want);
            int hit = -1, last = -1;  // (the vector's sum was rounded: the last with weight, should none reach the point)
            u64 run = before + up_to - own;
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (w[e] > 0.f) {
                    last = pos + e;
                    run += units_of(w[e]);
                    if (hit < 0 && run > want) hit = pos + e;
                }
            if (above) token = __shfl_sync(~0u, hit >= 0 ? hit : last, __ffs(above) - 1) - skip;
            before += __shfl_sync(~0u, up_to, 31);
        }
        if (lane == 0) drawn(token);
    } else if (chosen < 0 && part == 0 && lane == 0) {
        drawn(-1);
    }
    if (rank == 0) {
        for (int i = threadIdx.x; i <= a.drafts; i += kThreads)
            if (i != at) {
                out[i] = i < at ? tokens[i] : -1;
                if (logprob) logprob[i] = i < at ? log_p(elem<T>::to(target[i * a.target_row + tokens[i]]), (int)tokens[i], row_stat[i]) : -INFINITY;
            }
    }
    if (blocks > 1) cluster.sync();  // no block leaves while another reads its masses
}

// How the rows are cut: as many chunks as give all multiprocessors some, of 2,048 to 65,536 logits (what a block
// does besides is as much as 10 instructions a logit of 14,000).
struct Cut {
    int rows, chunks;
    size_t bytes;
};
Cut cut_for(int sms, int64_t requests, int drafts, bool known, int vocab) {
    Cut c;
    c.rows = known ? 2 * drafts + 1 : drafts + 1;
    int64_t chunks = (4 * (int64_t)sms + requests * c.rows - 1) / (requests * c.rows);
    const int64_t least = (vocab + 65535) / 65536, most = (vocab + 2047) / 2048;
    chunks = chunks < least ? least : chunks > most ? most : chunks;
    c.chunks = (int)chunks;
    c.bytes = sizeof(Stat) * (size_t)requests * c.rows * c.chunks;
    return c;
}

// How many clusters of `blocks` blocks of k_draw the device runs at once (0: it cannot be asked).
template <typename T> int clusters_at_once(int blocks) {
    static std::atomic<int> known[64][kMostCluster + 1];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < 64 && (n = known[dev][blocks].load(std::memory_order_relaxed))) return n;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = blocks, at.val.clusterDim.y = 1, at.val.clusterDim.z = 1;
    cfg.gridDim = dim3(blocks), cfg.blockDim = dim3(kThreads), cfg.attrs = &at, cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, k_draw<T>, &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    if (dev < 64) known[dev][blocks].store(n, std::memory_order_relaxed);
    return n;
}

template <typename T> int run(const sim_op_verify_t *a, const Cut &c, cudaStream_t st) {
    constexpr int N = Vec<T>::N;
    const int chunk_len = ((a->vocab + N - 1 + c.chunks - 1) / c.chunks + N - 1) / N * N;  // positions, which begin up to N - 1 before the row
    Stat *stats = (Stat *)a->workspace;
    cudaError_t e = launch_early(k_rows<T>, (unsigned)(a->requests * (int64_t)c.rows * c.chunks), kThreads, 0, 1, st, *a, stats, c.rows, c.chunks, chunk_len);
    if (e != cudaSuccess) return launched("sim_op_verify (rows)", e);
    // as many blocks as run at once, of 4,096 logits at least.  (A cluster has its place within a part of the device: 37 of 8
    // blocks do not all find one where 296 blocks would, and took 23.8 us, of 4 19.4; 64 of 4 do, and take 50.1, of 2 61.4.)
    int blocks = 1;
    while (blocks < kMostCluster && a->vocab > blocks * 4096 && a->requests <= clusters_at_once<T>(2 * blocks)) blocks *= 2;
    const int step = 32 * N, parts = blocks * kWarps, stretch = ((a->vocab + N - 1 + parts - 1) / parts + step - 1) / step * step;
    e = launch_early(k_draw<T>, (unsigned)(a->requests * (int64_t)blocks), kThreads, 0, blocks, st, *a, (const Stat *)stats, c.rows, c.chunks, stretch);
    return launched("sim_op_verify (draw)", e);
}

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" size_t sim_op_verify_workspace(int32_t requests, int32_t drafts, int32_t with_draft, int32_t vocab) {
    if (requests < 1 || drafts < 0 || drafts > SIM_OP_MAX_DRAFTS || vocab < 1 || vocab > SIM_OP_MAX_VOCAB) return 256;
    const int sms = sm_count();
    if (!sms) return 0;
    const size_t n = cut_for(sms, requests, drafts, with_draft && drafts, vocab).bytes;
    return n < 256 ? 256 : n;
}

extern "C" int sim_op_verify(const sim_op_verify_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16 && a->type != SIM_OP_FP32) return fail(SIM_ERR_ARG, "unknown element type %d", a->type);
    if (a->requests < 0) return fail(SIM_ERR_ARG, "requests must not be negative");
    if (a->drafts < 0 || a->drafts > SIM_OP_MAX_DRAFTS) return fail(SIM_ERR_ARG, "a request has 0 to %d drafted tokens", SIM_OP_MAX_DRAFTS);
    if (a->vocab < 1 || a->vocab > SIM_OP_MAX_VOCAB) return fail(SIM_ERR_ARG, "a vocabulary has 1 to %d tokens", SIM_OP_MAX_VOCAB);
    if (a->requests == 0) return SIM_OK;
    if (a->requests > (1 << 24)) return fail(SIM_ERR_ARG, "a call has at most 2^24 requests");
    if (!a->target || !a->uniform || !a->out || !a->count || (!a->tokens && a->drafts))
        return fail(SIM_ERR_ARG, "target, tokens, uniform, out and count must not be NULL");
    if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < 256)
        return fail(SIM_ERR_ARG, "a workspace aligned to 256 bytes is needed");
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const Cut c = cut_for(sms, a->requests, a->drafts, a->draft && a->drafts, a->vocab);
    if ((int64_t)a->requests * c.rows * c.chunks > INT32_MAX)
        return fail(SIM_ERR_ARG, "requests * rows is too large");
    if (a->workspace_bytes < c.bytes) return fail(SIM_ERR_ARG, "the workspace must have %zu bytes", c.bytes);
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) return run<__nv_bfloat16>(a, c, st);
    return a->type == SIM_OP_FP16 ? run<__half>(a, c, st) : run<float>(a, c, st);
}
