// sample.cu -- one token per row of logits (mtsim_ops.h).
#include "ops.cuh"

#include <cmath>
#include <cooperative_groups.h>

namespace mtop {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

// A row belongs to a cluster of 1 to 8 blocks, each of which holds a part of it
// in shared memory, so that the row is read from memory once however many
// passes the limits take; sums and histograms meet in distributed shared memory.
// Bound by instructions (about 20 a logit) and a chain of a dozen cluster barriers,
// not by memory: 64 x 131,075 bfloat16 take 39.5 us (17 MB), 1 x 32,000 floats 16 us.
//
// Weights are whole numbers of 2^-40: their sums are exact, so neither the
// order of the additions nor the split over threads and blocks changes a
// result, and a threshold that is searched for is found exactly.
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kCoarse = 4096;  // bins of the first, approximate histogram
constexpr int kFine = 256;     // bins of an exact one
constexpr int kList = 1024;    // candidates for a threshold
constexpr int kFew = 128;      // so few that each is compared with all
constexpr int kBinsEach = kCoarse / kThreads;
constexpr float kUnit = 1099511627776.f, kUnitLog2 = 40.f;
constexpr int kMostCluster = 8;
constexpr int kMostStaged = 180 * 1024;  // bytes of a block's part
constexpr int kHalfStaged = 72 * 1024;   // of one that leaves room for another block

// Order-preserving whole number of a logit (not NaN); -0 ranks with 0.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// 2^x to about 2^-22 of itself: a weight above 2^-18 of the largest is off by
// more units of 2^-40 than one, others by none or one.
__device__ __forceinline__ float exp2_near(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A weight x <= 2^40 cut into x = 2^18 hi + lo by additions of 2^23 (whose
// sums' low bits are the whole number), because conversions to 64 bits run at a
// fraction of the rate.  The sums keep the constant, which is taken out at the end; 32
// bits hold 1,023 of each.
struct Cut {
    uint32_t hi, lo;
    __device__ __forceinline__ explicit Cut(float x) {
        const float t = __fmaf_rz(x, 3.814697265625e-06f, 8388608.f);
        hi = __float_as_uint(t), lo = __float_as_uint(fmaf(t - 8388608.f, -262144.f, x) + 8388608.f);
    }
    __device__ __forceinline__ u64 units() const { return ((u64)(hi - 0x4B000000u) << 18) + (lo - 0x4B000000u); }
};
struct Mass {
    uint32_t hi = 0, lo = 0, n = 0;
    __device__ __forceinline__ void add(const Cut &c) { hi += c.hi, lo += c.lo, ++n; }
    __device__ __forceinline__ void add_if(bool yes, const Cut &c) { hi += yes ? c.hi : 0, lo += yes ? c.lo : 0, n += yes; }
    __device__ __forceinline__ u64 units() const { return ((u64)(hi - n * 0x4B000000u) << 18) + (lo - n * 0x4B000000u); }
};

// floor(x * f), or the next whole number above with `up`, for 0 <= f < 1 (else 0 or x), without 64-bit floats.
__device__ __forceinline__ u64 share_of(u64 x, float f, bool up) {
    if (!(f > 0.f)) return 0;
    if (f >= 1.f) return x;
    const uint32_t b = __float_as_uint(f), e = b >> 23, m = (b & 0x7FFFFF) | (e ? 0x800000 : 0);
    const int shift = 150 - (e ? e : 1);  // f = m / 2^shift, shift >= 24
    const u64 lo = x * m, hi = __umul64hi(x, m);
    u64 whole;
    bool rest;
    if (shift < 64) whole = hi << (64 - shift) | lo >> shift, rest = lo << (64 - shift);
    else whole = shift < 128 ? hi >> (shift - 64) : 0, rest = lo || (whole << (shift - 64)) != hi || shift >= 128;
    return whole + (up && rest);
}

struct Weights {
    float top, per;  // the largest logit, log2(e) / temperature
    __device__ __forceinline__ float of(float v) const { return exp2_near(fmaf(v - top, per, kUnitLog2)); }  // in units
    __device__ __forceinline__ u64 units(float v) const { return Cut(of(v)).units(); }
};

struct Sums {
    u64 mass, mass2;
    uint32_t count, high;
};

// What the blocks of a cluster read of each other; two of each, used in turn,
// so that one barrier a pass is enough.
struct Shared {
    union {
        uint32_t coarse[kCoarse];
        struct {  // candidates of the whole cluster
            uint32_t key[2][kList];
            u64 unit[kList];
        } all;
    };
    uint32_t list[2][kList], place[2][kList], listed[2];  // candidates of this block, by count and by weight: keys, positions
    uint32_t count[2][kFine], low[2][kFine], high[2][kFine];  // mass in two words
    Sums sums[2];
    // the block's own
    u64 warp_mass[kWarps], warp_mass2[kWarps];
    uint32_t warp_count[kWarps];
    u64 scan_mass[kWarps];
    uint32_t scan_count[kWarps];
    uint32_t found[4];
    u64 found_mass[2];
    u64 rank_mass[2][kMostCluster];  // what each block summed in the last exchange
    u64 rank_kept[kMostCluster];
    uint32_t rank_ties[kMostCluster];
    u64 warp_base[kWarps];
    uint32_t warp_hi[kWarps], warp_lo[kWarps];
    float found_real[1];
};

__device__ __forceinline__ u64 shfl_up64(u64 v, int o) { return __shfl_up_sync(~0u, v, o); }

template <typename V> __device__ __forceinline__ V warp_total(V v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

template <typename T> struct Part {
    static constexpr int N = 16 / sizeof(T);
    const T *row;    // the row's first logit, `skip` elements after a 16-byte boundary
    const T *held;   // the part in shared memory, or NULL
    int skip, vocab, begin, warp_len;  // positions count from that boundary
    bool endless;    // the largest logit is +infinity: it counts as 0, all others as -infinity
    __device__ __forceinline__ float value(T x) const {
        const float v = fmaxf(elem<T>::to(x), -INFINITY);  // NaN: -infinity
        return !endless ? v : v == INFINITY ? 0.f : -INFINITY;
    }

    // 16 bytes of the part from position p on (relative to it), -infinity where the row is not
    __device__ __forceinline__ void global(int p, T *x) const {
        const int i = begin + p - skip;
        if (i >= 0 && i + N <= vocab) {
            *(uint4 *)x = *(const uint4 *)(row + i);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = i + e >= 0 && i + e < vocab ? row[i + e] : elem<T>::from(-INFINITY);
        }
    }
    // The N logits at position p of the part.
    __device__ __forceinline__ void at(int p, float *v) const {
        alignas(16) T x[N];
        if (held) *(uint4 *)x = *(const uint4 *)(held + p);
        else global(p, x);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = value(x[e]);
    }
    // f(position, logits) over this warp's stretch, in vocabulary order: lane by lane within a step
    template <typename F> __device__ __forceinline__ void each(F f) const {
        const int lane = threadIdx.x % 32, from = threadIdx.x / 32 * warp_len;
        for (int p = from + lane * N; p < from + warp_len; p += 32 * N) {
            float v[N];
            at(p, v);
            f(p, v);
        }
    }
};

template <typename T> __global__ void __launch_bounds__(kThreads, 2) k_sample(const __grid_constant__ sim_op_sample_t a, int warp_len, bool staged, int bins) {
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t row = blockIdx.x / blocks;
    // a bin of one representable value: the bits of a key below it are the same for every logit of the type
    constexpr int kGrain = sizeof(T) == 4 ? 0 : std::is_same<T, __half>::value ? 13 : 16;

    Part<T> part;
    part.row = (const T *)a.logits + row * a.logits_row;
    part.skip = (int)(((uintptr_t)part.row & 15) / sizeof(T));
    part.vocab = a.vocab;
    part.warp_len = warp_len;
    part.begin = rank * warp_len * kWarps;
    part.held = nullptr, part.endless = false;
    T *const mine = (T *)dynamic;

    let_next_start();
    after_previous();
    int turn = 0;  // which of the two exchange buffers
    auto barrier = [&]() {
        if (blocks > 1) cluster.sync();
        else __syncthreads();
    };
    auto peer = [&](auto *p, int r) { return blocks > 1 ? cluster.map_shared_rank(p, r) : p; };

    // ------------------------------------------------ the row, its largest logit
    float high = -INFINITY;
    {
        const int at = warp * warp_len;
        for (int p = at + lane * Part<T>::N; p < at + warp_len; p += 32 * Part<T>::N) {
            alignas(16) T x[Part<T>::N];
            part.global(p, x);
            if (staged) *(uint4 *)(mine + p) = *(const uint4 *)x;
#pragma unroll
            for (int e = 0; e < Part<T>::N; ++e) high = fmaxf(high, elem<T>::to(x[e]));
        }
        if (staged) part.held = mine;
    }
    for (int b = threadIdx.x; b < bins; b += kThreads) sh.coarse[b] = 0;
    if (threadIdx.x < 2) sh.listed[threadIdx.x] = 0;
    uint32_t best = __reduce_max_sync(~0u, key_of(high));
    if (lane == 0) sh.warp_count[warp] = best;
    __syncthreads();
    best = __reduce_max_sync(~0u, sh.warp_count[lane % kWarps]);
    if (threadIdx.x == 0) sh.sums[turn].high = best;
    barrier();
    best = __reduce_max_sync(~0u, *peer(&sh.sums[turn].high, lane % blocks));
    turn ^= 1;

    Weights w;
    w.top = value_of(best);
    if (w.top == INFINITY) part.endless = true, w.top = 0.f, best = key_of(0.f);
    const float t = a.temperature ? a.temperature[row] : 1.f;
    const bool greedy = !(t > 0);
    w.per = fminf(fmaxf(1.4426950408889634f / t, 1.2e-38f), 3e38f);  // not 0 or infinite: -infinity * 0 and 0 * infinity are NaN
    const int k = a.top_k ? a.top_k[row] : 0;
    const float p = a.top_p ? a.top_p[row] : 1.f;
    // min_p in units; the largest logit always stays
    const float least = a.min_p ? fminf(a.min_p[row], 1.f) * kUnit : 0.f;
    const bool limit_k = !greedy && k > 0 && k < a.vocab, limit_p = !greedy && p < 1.f;

    // Sum over the block, then over the cluster: every thread gets the total.
    auto total_of = [&](u64 mass, u64 mass2, uint32_t count, Sums &out, Sums *before) {
        mass = warp_total(mass), mass2 = warp_total(mass2), count = __reduce_add_sync(~0u, count);
        if (lane == 0) sh.warp_mass[warp] = mass, sh.warp_mass2[warp] = mass2, sh.warp_count[warp] = count;
        __syncthreads();
        if (warp == 0) {
            const bool real = lane < kWarps;
            const u64 m = warp_total(real ? sh.warp_mass[lane] : 0), m2 = warp_total(real ? sh.warp_mass2[lane] : 0);
            const uint32_t c = __reduce_add_sync(~0u, real ? sh.warp_count[lane] : 0);
            if (lane == 0) sh.sums[turn].mass = m, sh.sums[turn].mass2 = m2, sh.sums[turn].count = c;
        }
        barrier();
        // a lane a block
        const Sums *from = peer(&sh.sums[turn], lane % blocks);
        const bool real = lane < blocks;
        const u64 m = real ? from->mass : 0, m2 = real ? from->mass2 : 0;
        const uint32_t c = real ? from->count : 0;
        out.mass = warp_total(m), out.mass2 = warp_total(m2), out.count = __reduce_add_sync(~0u, c);
        if (before) {
            before->mass = warp_total(lane < rank ? m : 0);
            before->count = __reduce_add_sync(~0u, lane < rank ? c : 0);
        }
        turn ^= 1;
    };

    bool listed = false;  // `bound` was found among the candidates, of which each block has all
    // kept: keys above `bound`, and the first `ties` (in vocabulary order) of the `equal` ones that have it
    uint32_t bound = 0, ties = 0, equal = 0;
    if (w.top == -INFINITY) {
        if (rank == 0 && threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        barrier();
        return;
    }
    if (greedy) bound = best, ties = 1, equal = 2;  // the first of them

    if (limit_k || limit_p) {
        // ------------------------------ where to look: counts over 41 powers of two of weight
        const float fine = (bins - 1) / 41.f, slope = fminf(w.per * fine, 3e38f), last_bin = (float)(bins - 1);
        part.each([&](int, const float *v) {
#pragma unroll
            for (int e = 0; e < Part<T>::N; ++e) {
                const uint32_t bin = __float_as_uint(fminf((w.top - v[e]) * slope, last_bin) + 8388608.f) & 0xFFFF;
                if (v[e] > -INFINITY) atomicAdd(&sh.coarse[bin], 1u);
            }
        });
        barrier();
        // Sums of the blocks' bins: each block adds up its share of the bins (in
        // place: no other reads those of it) and then all take every share.
        const int share = bins / blocks;
        if (blocks > 1) {
            for (int b = rank * share + threadIdx.x; b < (rank + 1) * share; b += kThreads) {
                uint32_t c = 0;
#pragma unroll 4
                for (int q = 0; q < blocks; ++q) c += *peer(&sh.coarse[b], (rank + q) % blocks);
                sh.coarse[b] = c;
            }
            barrier();
        }
        // a thread has some neighbouring bins; counts and approximate weight up to and with them
        const int each_bins = bins / kThreads, first_bin = each_bins * threadIdx.x;
        uint32_t bin_count[kBinsEach] = {};
        {
            const uint32_t *from = peer(&sh.coarse[first_bin], first_bin / share);
            if (each_bins == 8) {
                const uint4 c = *(const uint4 *)from, d = *(const uint4 *)(from + 4);
                bin_count[0] = c.x, bin_count[1] = c.y, bin_count[2] = c.z, bin_count[3] = c.w;
                bin_count[4] = d.x, bin_count[5] = d.y, bin_count[6] = d.z, bin_count[7] = d.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < each_bins) bin_count[e] = from[e];
            }
        }
        auto bin_weight = [&](int bin) { return exp2_near(40.f - bin / fine); };  // bins are about their middles
        uint32_t counts = 0;
        float masses = 0.f;
#pragma unroll
        for (int e = 0; e < kBinsEach; ++e) counts += bin_count[e], masses += bin_count[e] * bin_weight(first_bin + e);
        uint32_t prior_count = counts;
        float prior_mass = masses;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(~0u, counts, o);
            const float f = __shfl_up_sync(~0u, masses, o);
            if (lane >= o) counts += u, masses += f;
        }
        if (lane == 31) sh.scan_count[warp] = counts, sh.warp_count[warp] = __float_as_uint(masses);
        __syncthreads();
        {
            uint32_t cw = lane < kWarps ? sh.scan_count[lane] : 0;
            float mw = lane < kWarps ? __uint_as_float(sh.warp_count[lane]) : 0.f;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(~0u, cw, o);
                const float f = __shfl_up_sync(~0u, mw, o);
                if (lane >= o) cw += u, mw += f;
            }
            prior_count = counts - prior_count, prior_mass = masses - prior_mass;
            if (warp > 0) {
                prior_count += __shfl_sync(~0u, cw, warp - 1);
                prior_mass += __shfl_sync(~0u, mw, warp - 1);
            }
            masses = __shfl_sync(~0u, mw, 31);  // all of it
        }
        // The bin in which a count or a weight is reached, as keys with a bin to
        // spare on both sides; and the weight above it with as much of it as the count takes.
        auto look = [&](bool by_mass, uint32_t want, float want_mass, uint32_t &lo, uint32_t &hi, float &to_there) {
            __syncthreads();
            if (threadIdx.x == 0) sh.found[0] = bins;
            __syncthreads();
            uint32_t c = prior_count;
            float m = prior_mass;
#pragma unroll
            for (int e = 0; e < kBinsEach; ++e) {
                const int bin = first_bin + e;
                const float bw = bin_weight(bin), m2 = m + bin_count[e] * bw;
                const uint32_t c2 = c + bin_count[e];
                if (by_mass ? m < want_mass && m2 >= want_mass : c < want && c2 >= want) {
                    if (atomicMin(&sh.found[0], (uint32_t)bin) > (uint32_t)bin && !by_mass) sh.found_real[0] = m + (want - c) * bw;
                }
                c = c2, m = m2;
            }
            __syncthreads();
            const int bin = (int)sh.found[0];
            to_there = bin < bins ? sh.found_real[0] : masses;
            hi = best, lo = 0;
            if (bin < bins) {
                if (bin > 1) hi = min(best, key_of(w.top - (bin - 1.5f) / slope));
                if (bin < bins - 2) lo = key_of(w.top - (bin + 1.5f) / slope);
                if (lo > hi) lo = 0;
            }
        };
        // The key at which the count (or the weight) of the logits from the
        // largest down reaches `want`: exact histograms of ever narrower ranges of keys.
        auto search = [&](bool by_mass, u64 want, uint32_t lo, uint32_t hi, Sums &over, uint32_t &at, uint32_t &same) {
            for (int guard = 0; guard < 64; ++guard) {
                int shift = kGrain;
                while (((hi >> shift) - (lo >> shift)) >= kFine) ++shift;
                const uint32_t base = lo >> shift;
                const int n = (int)((hi >> shift) - base) + 1;
                for (int b = threadIdx.x; b < kFine; b += kThreads) sh.count[turn][b] = sh.low[turn][b] = sh.high[turn][b] = 0;
                __syncthreads();
                Mass mass;
                uint32_t count = 0;
                part.each([&](int, const float *v) {
#pragma unroll
                    for (int e = 0; e < Part<T>::N; ++e) {
                        const uint32_t key = key_of(v[e]), cell = key >> shift;
                        if (cell >= base + n) {
                            ++count;
                            if (by_mass) mass.add(Cut(w.of(v[e])));
                        } else if (cell >= base && v[e] > -INFINITY) {
                            atomicAdd(&sh.count[turn][cell - base], 1u);
                            if (by_mass) {
                                const u64 u = w.units(v[e]);
                                const uint32_t lw = (uint32_t)u, old = atomicAdd(&sh.low[turn][cell - base], lw);
                                const uint32_t hw = (uint32_t)(u >> 32) + (old + lw < old);
                                if (hw) atomicAdd(&sh.high[turn][cell - base], hw);
                            }
                        }
                    }
                });
                const int used = turn;
                total_of(mass.units(), 0, count, over, nullptr);
                // thread b has the b-th bin from the top
                uint32_t c = 0;
                u64 m = 0;
                if ((int)threadIdx.x < n) {
                    const int b = n - 1 - threadIdx.x;
                    for (int r = 0; r < blocks; ++r) {
                        c += *peer(&sh.count[used][b], r);
                        if (by_mass) m += *peer(&sh.low[used][b], r) + ((u64)*peer(&sh.high[used][b], r) << 32);
                    }
                }
                uint32_t ci = c;
                u64 mi = m;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t u = __shfl_up_sync(~0u, ci, o);
                    const u64 f = shfl_up64(mi, o);
                    if (lane >= o) ci += u, mi += f;
                }
                if (lane == 31) sh.scan_count[warp] = ci, sh.scan_mass[warp] = mi;
                if (threadIdx.x == 0) sh.found[1] = kFine;
                __syncthreads();
                for (int q = 0; q < warp && q < kFine / 32; ++q) ci += sh.scan_count[q], mi += sh.scan_mass[q];
                const u64 got = by_mass ? over.mass + mi : over.count + (u64)ci, prior = by_mass ? got - m : got - c;
                if ((int)threadIdx.x < n && got >= want && prior < want) {
                    sh.found[1] = n - 1 - threadIdx.x;
                    sh.found[2] = over.count + ci - c, sh.found[3] = c;
                    sh.found_mass[0] = over.mass + mi - m;
                }
                __syncthreads();
                const u64 above = by_mass ? over.mass : over.count;
                const uint32_t b = sh.found[1];
                if (above >= want) {  // the range was below it
                    lo = (base + n) << shift, hi = best;
                    continue;
                }
                if (b == kFine) {  // or above it; with nothing below, everything is kept
                    if (base == 0) {
                        at = 0, same = 0;
                        return;
                    }
                    hi = (base << shift) - 1, lo = 0;
                    continue;
                }
                over.count = sh.found[2], over.mass = sh.found_mass[0];
                const uint32_t first = (base + b) << shift;
                if (shift == kGrain) {
                    const uint32_t low_bits = (1u << kGrain) - 1;
                    at = first & 0x80000000u ? first : first | low_bits;
                    same = sh.found[3];
                    return;
                }
                lo = first, hi = min(best, first + ((1u << shift) - 1));
                __syncthreads();
            }
            at = 0, same = 0;
        };

        // Candidates: the logits in the bins where the thresholds lie, and the
        // exact count and weight of those above them.
        uint32_t lo_k = 0, hi_k = 0, lo_p = 0, hi_p = 0;
        float to_k = 0.f, unused;
        if (limit_k) look(false, (uint32_t)k, 0.f, lo_k, hi_k, to_k);
        else to_k = masses;
        if (limit_p) look(true, 0, fmaxf(p, 0.f) * to_k, lo_p, hi_p, unused);
        Sums over;
        {
            Mass m1, m2;  // of all (of those above the count's candidates), of those above the weight's
            uint32_t count = 0;
            // (comparisons of logits: a key is only made of a candidate)
            auto floor_of = [&](uint32_t key) { return key ? value_of(key) : -INFINITY; };
            const float top_k = limit_k ? value_of(hi_k) : 0.f, low_k = floor_of(lo_k), top_p = limit_p ? value_of(hi_p) : 0.f, low_p = floor_of(lo_p);
            auto list = [&](int l, float v, int pos) {
                const uint32_t at = atomicAdd(&sh.listed[l], 1u);
                if (at < kList) sh.list[l][at] = key_of(v), sh.place[l][at] = pos;
            };
            if (limit_k) {
                // What is below all candidates adds to nothing: most steps of a warp skip
                // the rest (64 x 131,075, k = 1,000 32.5 us; without 36.4).
                const float lowest = limit_p ? fminf(low_k, low_p) : low_k;
                part.each([&](int pos, const float *v) {
#pragma unroll
                    for (int e = 0; e < Part<T>::N; ++e) {
                        if (!__any_sync(~0u, v[e] >= lowest)) continue;
                        const Cut x(w.of(v[e]));
                        const bool above = v[e] > top_k;
                        m1.add_if(above, x);
                        count += above;
                        if (!above && v[e] >= low_k) list(0, v[e], pos + e);
                        if (limit_p) {
                            const bool above_p = v[e] > top_p;
                            m2.add_if(above_p, x);
                            if (!above_p && v[e] >= low_p) list(1, v[e], pos + e);
                        }
                    }
                });
            } else {
                part.each([&](int pos, const float *v) {
#pragma unroll
                    for (int e = 0; e < Part<T>::N; ++e) {
                        const Cut x(w.of(v[e]));
                        const bool above = v[e] > top_p;
                        m1.add(x);
                        m2.add_if(above, x);
                        if (!above && v[e] >= low_p) list(1, v[e], pos + e);
                    }
                });
            }
            total_of(m1.units(), m2.units(), count, over, nullptr);
            if (threadIdx.x < blocks) {
                const Sums *from = peer(&sh.sums[turn ^ 1], threadIdx.x);
                sh.rank_mass[0][threadIdx.x] = from->mass, sh.rank_mass[1][threadIdx.x] = from->mass2;
            }
            if (threadIdx.x < kWarps) {
                sh.warp_base[threadIdx.x] = limit_p ? sh.warp_mass2[threadIdx.x] : sh.warp_mass[threadIdx.x];
                sh.warp_hi[threadIdx.x] = sh.warp_lo[threadIdx.x] = 0;
            }
        }
        // every block takes the candidates of all: a warp a block's list
        int n_of[2];
#pragma unroll
        for (int l = 0; l < 2; ++l) {
            const uint32_t c = lane < blocks ? *peer(&sh.listed[l], lane % blocks) : 0;
            uint32_t end = c;
#pragma unroll
            for (int o = 1; o < kMostCluster; o <<= 1) {
                const uint32_t u = __shfl_up_sync(~0u, end, o);
                if (lane >= o) end += u;
            }
            const uint32_t n = __shfl_sync(~0u, end, blocks - 1);
            n_of[l] = n <= kList ? (int)n : -1;
            const int r = warp - l * kMostCluster;
            if (n <= kList && r >= 0 && r < blocks) {
                const uint32_t to = __shfl_sync(~0u, end - c, r), mine_of = __shfl_sync(~0u, c, r);
                const uint32_t *from = peer(&sh.list[l][0], r);
                for (uint32_t i = lane; i < mine_of; i += 32) {
                    const uint32_t key = from[i];
                    sh.all.key[l][to + i] = key;
                    if (l == limit_p) sh.all.unit[to + i] = w.units(value_of(key));
                }
            }
        }
        __syncthreads();
        // The threshold among the candidates: each warp tries a key at a time.  False if it is not among them (the bins are approximate) or they are too many.
        auto among = [&](bool by_mass, u64 want, u64 above, uint32_t lo, uint32_t hi, u64 &before, uint32_t &at, uint32_t &same) -> bool {
            const int l = by_mass, n = n_of[l];
            if (n < 0 || above >= want) return false;
            if (n <= kFew) {  // each candidate against all
                __syncthreads();
                if (threadIdx.x == 0) sh.found[1] = 0;
                __syncthreads();
                if ((int)threadIdx.x < n) {
                    const uint32_t key = sh.all.key[l][threadIdx.x];
                    u64 over = above;
                    uint32_t eq = 0;
                    for (int j = 0; j < n; ++j) {
                        const uint32_t other = sh.all.key[l][j];
                        if (other > key) over += by_mass ? sh.all.unit[j] : 1;
                        eq += other == key;
                    }
                    const u64 each = by_mass ? sh.all.unit[threadIdx.x] : 1;
                    if (over < want && over + eq * each >= want) sh.found[1] = 1, sh.found[2] = key, sh.found[3] = eq, sh.found_mass[0] = over;
                }
                __syncthreads();
                before = sh.found_mass[0], at = sh.found[2], same = sh.found[3];
                return sh.found[1] != 0;
            }
            uint32_t base = lo >> kGrain, size = (hi >> kGrain) - base + 1;  // the answer's cell lies in [base, base + size)
            before = above;
            for (bool first = true; first || size > 1; first = false) {
                const uint32_t step = (size + kWarps - 1) / kWarps, from = base + warp * step;
                u64 m = 0;  // of candidates in cells >= from
                if (warp * step < size)
                    for (int i = lane; i < n; i += 32)
                        if (sh.all.key[l][i] >> kGrain >= from) m += by_mass ? sh.all.unit[i] : 1;
                m = warp_total(m);
                __syncthreads();
                if (lane == 0) sh.scan_mass[warp] = warp * step < size ? above + m : 0;
                __syncthreads();
                const uint32_t reach = __ballot_sync(~0u, lane < kWarps && sh.scan_mass[lane % kWarps] >= want);
                if (!reach) return false;
                const int last = 31 - __clz(reach);
                // (cells from the next try on do not reach it)
                if (last + 1 < kWarps && (last + 1) * step < size) before = sh.scan_mass[last + 1];
                const uint32_t cut = base + last * step;
                size = min(step, size - last * step), base = cut;
            }
            // how many have that key
            uint32_t c = 0;
            for (int i = threadIdx.x; i < n; i += kThreads) c += sh.all.key[l][i] >> kGrain == base;
            c = __reduce_add_sync(~0u, c);
            if (lane == 0) sh.scan_count[warp] = c;
            __syncthreads();
            same = __reduce_add_sync(~0u, lane < kWarps ? sh.scan_count[lane] : 0);
            const uint32_t first = base << kGrain;
            at = first & 0x80000000u ? first : first | ((1u << kGrain) - 1);
            return same > 0;
        };

        const Sums gathered = over;
        u64 have = gathered.mass;
        if (limit_k) {
            u64 before;
            if (among(false, (u64)k, gathered.count, lo_k, hi_k, before, bound, equal)) {
                listed = true;
                ties = (uint32_t)(k - before);
                if (limit_p) {  // the weight that stays: above the candidates, and theirs
                    u64 m = 0;
                    for (int i = threadIdx.x; i < n_of[0]; i += kThreads) {
                        const uint32_t key = sh.all.key[0][i];
                        if (key > bound) m += w.units(value_of(key));
                    }
                    m = warp_total(m);
                    __syncthreads();
                    if (lane == 0) sh.scan_mass[warp] = m;
                    __syncthreads();
                    have = gathered.mass + warp_total(lane < kWarps ? sh.scan_mass[lane] : 0) + ties * w.units(value_of(bound));
                }
            } else {
                search(false, (u64)k, lo_k, hi_k, over, bound, equal);
                ties = bound ? (uint32_t)k - over.count : 0;
                if (limit_p) {
                    Mass m;
                    part.each([&](int, const float *v) {
#pragma unroll
                        for (int e = 0; e < Part<T>::N; ++e)
                            if (key_of(v[e]) > bound) m.add(Cut(w.of(v[e])));
                    });
                    total_of(m.units(), 0, 0, over, nullptr);
                    have = over.mass + (bound ? ties * w.units(value_of(bound)) : 0);
                }
            }
        }
        if (limit_p) {
            u64 want = share_of(have, p, true), before;
            if (want < 1) want = 1;
            uint32_t at, same;
            listed = among(true, want, gathered.mass2, lo_p, hi_p, before, at, same);
            if (!listed) {
                search(true, want, lo_p, hi_p, over, at, same);
                before = over.mass;
            }
            if (at && at >= bound) {
                const u64 unit = w.units(value_of(at));
                const u64 need = unit ? (want - before + unit - 1) / unit : 1;
                const uint32_t room = at == bound ? ties : same;
                bound = at, equal = same, ties = need < room ? (uint32_t)need : room;
            }
        }
    }

    const float cut_at = bound ? value_of(bound) : -INFINITY;
    auto kept = [&](float v, int pos, int last) -> float {
        if (!(v >= cut_at) || (bound && v == cut_at && pos > last)) return 0.f;
        if (greedy) return 1.f;
        const float x = w.of(v);
        return x < least ? 0.f : x;
    };
    const float u = a.uniform[row];
    // The draw within the stretch of warp `owner`, `ahead` being the kept weight
    // before it: every warp of the block takes one of its steps at a time.
    auto draw = [&](int owner, u64 ahead, u64 target, u64 total, int last) {
        constexpr int step = 32 * Part<T>::N;
        for (int first = 0; first < warp_len; first += kWarps * step) {
            const int p = owner * warp_len + first + warp * step + lane * Part<T>::N;
            const bool in = first + warp * step < warp_len;
            float v[Part<T>::N];
            u64 x[Part<T>::N], sum = 0;
            if (in) part.at(p, v);
#pragma unroll
            for (int e = 0; e < Part<T>::N; ++e) x[e] = in ? Cut(kept(v[e], p + e, last)).units() : 0, sum += x[e];
            u64 incl = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 up = shfl_up64(incl, o);
                if (lane >= o) incl += up;
            }
            __syncthreads();
            if (lane == 31) sh.scan_mass[warp] = incl;
            __syncthreads();
            u64 at = ahead + incl - sum;
            for (int q = 0; q < kWarps; ++q) {
                if (q < warp) at += sh.scan_mass[q];
                ahead += sh.scan_mass[q];
            }
#pragma unroll
            for (int e = 0; e < Part<T>::N; ++e) {
                if (x[e] && at <= target && at + x[e] > target) {
                    a.token[row] = part.begin + p + e - part.skip;
                    if (a.logprob) {
                        const float share = (float)((double)total * (1.0 / (double)kUnit));
                        a.logprob[row] = greedy ? 0.f : (v[e] - w.top) / t - logf(share);
                    }
                }
                at += x[e];
            }
        }
    };
    auto target_of = [&](u64 total) {
        const u64 at = share_of(total, u, false);
        return at < total ? at : total - 1;
    };

    if (listed && !(w.of(value_of(bound)) < least)) {
        // ---------- the draw from the sums above the candidates and the candidates that stay:
        // every block finds the block that has it, and that one the warp, without another pass
        const int l = limit_p;
        const u64 unit = w.units(value_of(bound));
        if (warp < blocks) {
            uint32_t from = 0;
            const uint32_t each = lane < blocks ? *peer(&sh.listed[l], lane % blocks) : 0;
            from = __reduce_add_sync(~0u, lane < warp ? each : 0);
            const uint32_t n = __shfl_sync(~0u, each, warp);
            u64 m = 0;
            uint32_t c = 0;
            for (uint32_t i = lane; i < n; i += 32) {
                const uint32_t key = sh.all.key[l][from + i];
                if (key > bound) m += sh.all.unit[from + i];
                c += key == bound;
            }
            m = warp_total(m), c = __reduce_add_sync(~0u, c);
            if (lane == 0) sh.rank_kept[warp] = sh.rank_mass[l][warp] + m, sh.rank_ties[warp] = c;
        }
        __syncthreads();
        u64 total = 0;
        uint32_t left = ties;
        for (int r = 0; r < blocks; ++r) {
            const uint32_t c = min(left, sh.rank_ties[r]);
            total += sh.rank_kept[r] + c * unit, left -= c;
        }
        const u64 target = target_of(total);
        u64 ahead = 0;
        uint32_t stay = 0;
        bool here = false;
        left = ties;
        for (int r = 0; r <= rank; ++r) {
            stay = min(left, sh.rank_ties[r]);
            const u64 has = sh.rank_kept[r] + stay * unit;
            left -= stay;
            here = target >= ahead && target - ahead < has;
            if (r < rank) ahead += has;
        }
        if (here) {
            if (threadIdx.x == 0) sh.found[0] = stay < sh.rank_ties[rank] ? 0 : 1u << 30;
            __syncthreads();
            const uint32_t n = sh.listed[l];
            for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
                const uint32_t key = sh.list[l][i], pos = sh.place[l][i];
                bool stays = key > bound;
                if (key == bound) {
                    uint32_t before = 0;  // equal ones before it
                    if (stay < sh.rank_ties[rank])
                        for (uint32_t j = 0; j < n; ++j) before += sh.list[l][j] == bound && sh.place[l][j] < pos;
                    stays = before < stay;
                    if (stays && stay < sh.rank_ties[rank]) atomicMax(&sh.found[0], pos + 1);
                }
                if (stays) {
                    const u64 x = w.units(value_of(key));
                    atomicAdd(&sh.warp_hi[pos / part.warp_len], (uint32_t)(x >> 18));
                    atomicAdd(&sh.warp_lo[pos / part.warp_len], (uint32_t)x & 0x3FFFF);
                }
            }
            __syncthreads();
            auto of_warp = [&](int q) { return sh.warp_base[q] + ((u64)sh.warp_hi[q] << 18) + sh.warp_lo[q]; };
            int owner = 0;
            for (; owner + 1 < kWarps; ++owner) {
                const u64 own = of_warp(owner);
                if (target - ahead < own) break;
                ahead += own;
            }
            draw(owner, ahead, target, total, (int)sh.found[0] - 1);
        }
        barrier();  // no block leaves while another may read its shared memory
        return;
    }

    // ------------------------------------- equal ones: which of them stay
    int last_tie = 1 << 30;  // the position in this part of the last one that stays
    if (bound && ties < equal) {
        uint32_t n = 0;
        part.each([&](int, const float *v) {
#pragma unroll
            for (int e = 0; e < Part<T>::N; ++e) n += key_of(v[e]) == bound;
        });
        const uint32_t of_warp = warp_total(n);
        Sums all, before;
        total_of(0, 0, n, all, &before);
        if (before.count >= ties) last_tie = -1;
        else {
            uint32_t ahead = before.count;  // of this warp's stretch
            for (int q = 0; q < warp; ++q) ahead += sh.warp_count[q];
            if (threadIdx.x == 0) sh.found[0] = 1u << 30;
            __syncthreads();
            if (ahead < ties && ahead + of_warp >= ties) {
                part.each([&](int pos, const float *v) {
                    const uint32_t active = __activemask();
                    uint32_t c = 0;
#pragma unroll
                    for (int e = 0; e < Part<T>::N; ++e) c += key_of(v[e]) == bound;
                    uint32_t incl = c;
                    for (int o = 1; o < 32; o <<= 1) {
                        const uint32_t u = __shfl_up_sync(active, incl, o);
                        if (lane >= o) incl += u;
                    }
                    uint32_t rank_of = ahead + incl - c;
#pragma unroll
                    for (int e = 0; e < Part<T>::N; ++e)
                        if (key_of(v[e]) == bound && ++rank_of == ties) sh.found[0] = pos + e;
                    ahead += __shfl_sync(active, incl, 31);
                });
            }
            __syncthreads();
            last_tie = (int)sh.found[0];
        }
    }

    // -------------------------------------------------------------- the draw
    Mass m;
    part.each([&](int pos, const float *v) {
#pragma unroll
        for (int e = 0; e < Part<T>::N; ++e) m.add(Cut(kept(v[e], pos + e, last_tie)));
    });
    Sums all, before;
    total_of(m.units(), 0, 0, all, &before);
    const u64 target = target_of(all.mass);
    u64 ahead = before.mass;
    int owner = 0;
    bool here = target >= ahead;
    for (; here && owner < kWarps; ++owner) {
        const u64 own = sh.warp_mass[owner];
        if (target - ahead < own) break;
        ahead += own;
    }
    if (here && owner < kWarps) draw(owner, ahead, target, all.mass, last_tie);  // one block of the cluster
    barrier();  // no block leaves while another may read its shared memory
}

template <typename T> int run(const sim_op_sample_t *a, cudaStream_t st) {
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    // Blocks a row: so many that two blocks' parts fit in a multiprocessor's shared
    // memory (128 x 131,075 bfloat16: 4 blocks 75 us, 2 blocks 86), and more while all
    // rows' blocks still run at once and a part is 2,048 logits or more (64 rows of
    // that: 4 blocks 39.5 us, 8 blocks 58; 64 x 32,000: 4 blocks 25.5 us, 1 block 44; 64 x
    // 8,000: 2 blocks 22.7 us, 4 blocks 23.2; 1 x 32,000: 8 blocks 16 us, 2 blocks 19.5).
    constexpr int N = 16 / sizeof(T);
    int blocks = 1;
    auto stretch = [&](int n) { return (int)(((int64_t)a->vocab + N - 1 + (int64_t)n * kWarps * 32 * N - 1) / ((int64_t)n * kWarps * 32 * N)) * 32 * N; };
    while (blocks < kMostCluster && (int64_t)stretch(blocks) * kWarps * (int)sizeof(T) > kHalfStaged) blocks *= 2;
    while (blocks < kMostCluster && (int64_t)a->rows * blocks * 2 <= 2 * sms && a->vocab / (blocks * 2) >= 2048) blocks *= 2;
    const int warp_len = stretch(blocks);
    const int64_t bytes = (int64_t)warp_len * kWarps * sizeof(T);
    const bool staged = bytes <= kMostStaged;
    static std::atomic<uint64_t> told;
    if (!allow_shared((const void *)k_sample<T>, kMostStaged, told)) return SIM_ERR_CUDA;
    int bins = kThreads;  // about 32 logits each
    while (bins < kCoarse && bins * 32 < a->vocab) bins *= 2;
    const cudaError_t e = launch_early(k_sample<T>, (unsigned)a->rows * blocks, kThreads, staged ? (size_t)bytes : 0, blocks, st, *a, warp_len, staged, bins);
    return launched("sim_op_sample", e);
}

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" int sim_op_sample(const sim_op_sample_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16 && a->type != SIM_OP_FP32) return fail(SIM_ERR_ARG, "unknown element type %d", a->type);
    if (a->rows < 0) return fail(SIM_ERR_ARG, "rows must not be negative");
    if (a->vocab < 1 || a->vocab > SIM_OP_MAX_VOCAB) return fail(SIM_ERR_ARG, "vocab must be in [1, %d]", SIM_OP_MAX_VOCAB);
    if (a->rows == 0) return SIM_OK;
    if (!a->logits || !a->uniform || !a->token) return fail(SIM_ERR_ARG, "logits, uniform and token must not be NULL");
    if (a->rows > INT32_MAX / kMostCluster) return fail(SIM_ERR_ARG, "rows must be below 2^28");
    const cudaStream_t st = (cudaStream_t)stream;
    return a->type == SIM_OP_BF16 ? run<__nv_bfloat16>(a, st) : a->type == SIM_OP_FP16 ? run<__half>(a, st) : run<float>(a, st);
}
