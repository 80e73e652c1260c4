// verify.cu -- which drafted tokens the target's probabilities keep, and the
// token that follows them (mtsim_ops.h).
#include "ops.cuh"

#include <cooperative_groups.h>

namespace mtop {
namespace {

namespace cg = cooperative_groups;

// Two kernels.  k_rows takes all rows of logits in chunks, a block a chunk, and leaves the chunk's largest logit
// and the sum of its weights.  k_draw, a cluster of blocks a request, joins these, decides how many tokens are
// accepted, goes once more over the one row (or the two) that the next token is drawn from (in L2 by then), and the
// warp whose stretch holds the point looks for it.
// Bound by memory, the row that is drawn from by instructions: MEASURED.
//
// Sums of a thread's and a warp's weights are in 32 bits, beyond that in 64 (which run at a
// sixtieth of the rate here): errors of single sums are independent, and those of 128 warps and more average out.
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBatch = 4;            // vectors that a thread has on their way
constexpr int kMostCluster = 8;

// log2(e) / t in two floats: (l - m) * (hi + lo) is the binary logarithm of a weight.  (Not zero for an infinite t:
// -infinity times it is -infinity.)
struct Rate {
    float hi, lo;
    bool greedy;
    __device__ explicit Rate(float t) {
        greedy = !(t > 0.f);
        const double r = greedy ? 0.0 : 1.4426950408889634 / (double)t;
        hi = fmaxf((float)r, 1e-36f), lo = hi < INFINITY && hi > 1e-36f ? (float)(r - (double)hi) : 0.f;
        hi = fminf(hi, 3e38f);
    }
};

__device__ __forceinline__ float exp2_near(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A chunk, or a whole row: its largest logit, the sum of the weights 2^(rate (l - top)), and the lowest index of
// the largest (greedy requests: all of the weight).
struct Stat {
    double sum;
    float top;
    int first;
};

// A weight to about 2^-22 of itself: the exponent's rounding (2^-24 of up to
// 126) is kept apart and multiplied in.
__device__ __forceinline__ float weight_of(float l, int v, float top, int first, const Rate &c) {
    if (c.greedy) return v == first ? 1.f : 0.f;
    if (!(l > -INFINITY)) return 0.f;  // (or NaN)
    if (top == INFINITY) return l == INFINITY ? 1.f : 0.f;
    const float d = __fsub_rn(l, top), b = __fsub_rn(d, l), off = __fsub_rn(__fsub_rn(l, __fsub_rn(d, b)), __fadd_rn(top, b));  // d + off = l - top
    const float y = __fmul_rn(d, c.hi);
    if (!(y > -126.f)) return 0.f;
    const float e = fmaf(d, c.hi, -y) + fmaf(d, c.lo, off * c.hi), p = exp2_near(y);
    return fmaf(p, e * 0.6931471805599453f, p);
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
__device__ __forceinline__ int warp_min(int v) { return __reduce_min_sync(~0u, v); }

// Logits v .. v + N - 1 of a row that begins anywhere (v < vocab), as they lie in one or two vectors of 16 bytes;
// results must not depend on where a row begins, so its vectors count from its first logit.
struct Raw {
    uint4 lo, hi;
};
template <typename T> __device__ __forceinline__ Raw fetch(const T *row, int v, int vocab) {
    const uintptr_t at = (uintptr_t)(row + v);
    const int shift = (int)(at & 15);
    const uint4 *from = (const uint4 *)(at - shift);
    Raw r;
    r.lo = from[0];
    // (the second holds an element of the row, or is not looked at)
    if (shift && v + (16 - shift) / (int)sizeof(T) < vocab) r.hi = from[1];
    return r;
}
// The same as 32-bit numbers, NaN and what lies past the row's end as -infinity.
template <typename T> __device__ __forceinline__ void logits_of(const Raw &r, const T *row, int v, int vocab, float *f) {
    constexpr int N = Vec<T>::N;
    const int shift = (int)((uintptr_t)(row + v) & 15);
    Vec<T> x;
    uint4 y = r.lo;
    if (shift) {
        uint32_t w[8] = {r.lo.x, r.lo.y, r.lo.z, r.lo.w, r.hi.x, r.hi.y, r.hi.z, r.hi.w};
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
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = fmaxf(f[e], -INFINITY);
    if (v + N > vocab) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (v + e >= vocab) f[e] = -INFINITY;
    }
}

// ------------------------------------------------------------- rows -------
template <typename T>
__global__ void __launch_bounds__(kThreads, 2) k_rows(const __grid_constant__ sim_op_verify_t a, Stat *stats, int rows, int chunks, int chunk_len) {
    constexpr int N = Vec<T>::N;
    __shared__ float tops[kWarps], sums[kWarps];
    __shared__ int firsts[kWarps];
    let_next_start();
    after_previous();
    const int64_t row = blockIdx.x / chunks, b = row / rows;
    const int chunk = (int)(blockIdx.x - row * chunks), k = (int)(row - b * rows), lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int drafted = a.drafted ? min(max(a.drafted[b], 0), a.drafts) : a.drafts;
    if (k <= a.drafts ? k > drafted : k - a.drafts - 1 >= drafted) return;  // of a token that is not there
    const T *from = k <= a.drafts ? (const T *)a.target + b * a.target_request + k * a.target_row
                                  : (const T *)a.draft + b * a.draft_request + (k - a.drafts - 1) * a.draft_row;
    const Rate c(a.temperature ? a.temperature[b] : 1.f);
    const int begin = chunk * chunk_len, end = min(begin + chunk_len, a.vocab);
    float top = -INFINITY, sum = 0.f;
    int first = 0x7FFFFFFF;
    for (int p0 = begin + threadIdx.x * N; p0 < end; p0 += kBatch * kThreads * N) {
        Raw v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (p0 + i * kThreads * N < end) v[i] = fetch(from, p0 + i * kThreads * N, a.vocab);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int p = p0 + i * kThreads * N;
            if (p >= end) break;
            float f[N];
            logits_of(v[i], from, p, a.vocab, f);
            float most = f[0];
#pragma unroll
            for (int e = 1; e < N; ++e) most = fmaxf(most, f[e]);
            if (c.greedy) {
                if (most > top) {
                    top = most;
#pragma unroll
                    for (int e = N - 1; e >= 0; --e)
                        if (f[e] == most) first = p + e;
                }
                continue;
            }
            if (most > top) {
                sum *= exp2_near((top - most) * c.hi);
                top = most;
                if (top == INFINITY) sum = 0.f;  // from here on only such count
            }
            if (top == INFINITY) {
#pragma unroll
                for (int e = 0; e < N; ++e) sum += f[e] == INFINITY;
            } else if (top > -INFINITY) {
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = f[e] - top;
                    part += exp2_near(fmaxf(fmaf(d, c.lo, d * c.hi), -200.f));  // (-infinity times lo may be anything)
                }
                sum += part;
            }
        }
    }
    const float high = warp_max(top);
    float s = top == -INFINITY ? 0.f : high == INFINITY ? (top == INFINITY ? sum : 0.f) : sum * exp2_near((top - high) * c.hi);
    s = warp_sum(s);
    first = warp_min(top == high ? first : 0x7FFFFFFF);
    if (lane == 0) tops[warp] = high, sums[warp] = s, firsts[warp] = first;
    __syncthreads();
    if (warp == 0) {
        const float t = lane < kWarps ? tops[lane] : -INFINITY, all = warp_max(t);
        const int f = warp_min(lane < kWarps && t == all ? firsts[lane] : 0x7FFFFFFF);
        double w = lane < kWarps && t > -INFINITY ? (t == all ? (double)sums[lane] : (double)(sums[lane] * exp2_near((t - all) * c.hi))) : 0.0;
#pragma unroll
        for (int o = kWarps / 2; o; o >>= 1) w += __shfl_xor_sync(~0u, w, o);
        if (lane == 0) stats[row * chunks + chunk] = {w, all, f};
    }
}

// ------------------------------------------------------------- draw -------
struct Peers {
    float mass[kWarps];  // of the block's warps' stretches
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) k_draw(const __grid_constant__ sim_op_verify_t a, const Stat *stats, int rows, int chunks, int stretch) {
    constexpr int N = Vec<T>::N;
    __shared__ Stat row_stat[2 * SIM_OP_MAX_DRAFTS + 1];
    __shared__ float log_of[SIM_OP_MAX_DRAFTS + 1];
    __shared__ bool passed[SIM_OP_MAX_DRAFTS];
    __shared__ Peers mine[2];
    __shared__ double ahead_of[kMostCluster * kWarps], whole;
    __shared__ int found;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t b = blockIdx.x / blocks;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    let_next_start();
    after_previous();
    const int drafted = a.drafted ? min(max(a.drafted[b], 0), a.drafts) : a.drafts;
    const Rate c(a.temperature ? a.temperature[b] : 1.f);
    const T *target = (const T *)a.target + b * a.target_request, *draft = a.draft ? (const T *)a.draft + b * a.draft_request : nullptr;
    const int64_t *tokens = a.tokens + b * a.drafts;
    const float *uniform = a.uniform + b * (a.drafts + 1);
    // the rows' chunks, a row a thread
    for (int k = threadIdx.x; k < rows; k += kThreads) {
        if (k <= a.drafts ? k > drafted : k - a.drafts - 1 >= drafted) continue;
        const Stat *s = stats + (b * rows + k) * chunks;
        Stat r = {0.0, -INFINITY, 0x7FFFFFFF};
        for (int i = 0; i < chunks; ++i) {
            const Stat x = s[i];
            if (x.top > r.top) r.top = x.top, r.first = x.first;
        }
        for (int i = 0; i < chunks; ++i) {
            const Stat x = s[i];
            if (x.top > -INFINITY) r.sum += x.top == r.top ? x.sum : r.top == INFINITY ? 0.0 : x.sum * (double)exp2_near((x.top - r.top) * c.hi);
        }
        if (c.greedy) r.sum = r.top > -INFINITY ? 1.0 : 0.0;
        row_stat[k] = r;
    }
    __syncthreads();
    auto log_p = [&](float l, int v, const Stat &p) {
        const float w = weight_of(l, v, p.top, p.first, c);
        if (!(w > 0.f)) return -INFINITY;
        if (c.greedy) return 0.f;
        return (float)(p.top == INFINITY ? -log(p.sum) : ((double)l - p.top) * ((double)c.hi + c.lo) * 0.6931471805599453 - log(p.sum));
    };
    // every drafted token's test, a token a thread
    if (threadIdx.x < drafted) {
        const int i = threadIdx.x;
        const int64_t x = tokens[i];
        const bool real = x >= 0 && x < a.vocab;
        const Stat p = row_stat[i];
        const float l = real ? elem<T>::to(target[i * a.target_row + x]) : -INFINITY;
        const double px = real && p.sum > 0.0 ? weight_of(l, (int)x, p.top, p.first, c) / p.sum : 0.0;
        double qx = real ? 1.0 : 0.0;
        if (draft && real) {
            const Stat q = row_stat[a.drafts + 1 + i];
            qx = q.sum > 0.0 ? weight_of(elem<T>::to(draft[i * a.draft_row + x]), (int)x, q.top, q.first, c) / q.sum : 0.0;
        }
        passed[i] = uniform[i] * qx < px;
        log_of[i] = passed[i] ? log_p(l, (int)x, p) : -INFINITY;
    }
    __syncthreads();
    int at = 0;
    while (at < drafted && passed[at]) ++at;
    // the row that is drawn from, a stretch a warp
    bool refused = at < drafted;
    const Stat p = row_stat[at], q = refused && draft ? row_stat[a.drafts + 1 + at] : Stat{1.0, 0.f, 0};
    const T *lp = target + at * a.target_row, *lq = refused && draft ? draft + at * a.draft_row : nullptr;
    const int64_t x = refused ? tokens[at] : -1;
    const float by_p = p.sum > 0.0 ? (float)(1.0 / p.sum) : 0.f, by_q = q.sum > 0.0 ? (float)(1.0 / q.sum) : 0.f;
    auto weights = [&](int v, float *w) {
        logits_of(fetch(lp, v, a.vocab), lp, v, a.vocab, w);
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = __fmul_rn(weight_of(w[e], v + e, p.top, p.first, c), by_p);
        if (!refused) return;
        if (lq) {
            float g[N];
            logits_of(fetch(lq, v, a.vocab), lq, v, a.vocab, g);
            // (two roundings and not one fused step: equal probabilities leave nothing)
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = fmaxf(__fsub_rn(w[e], __fmul_rn(weight_of(g[e], v + e, q.top, q.first, c), by_q)), 0.f);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (v + e == x) w[e] = fmaxf(__fsub_rn(w[e], 1.f), 0.f);
        }
    };
    const int part = rank * kWarps + warp, begin = part * stretch, end = min(begin + stretch, a.vocab);
    int chosen = -1;  // the part with the point
    double want = 0.0;
    for (int round = 0; round < 2; ++round) {
        float sum = 0.f;
        for (int v = begin + lane * N; v < end; v += 32 * N) {
            float w[N], s = 0.f;
            weights(v, w);
#pragma unroll
            for (int e = 0; e < N; ++e) s += w[e];
            sum += s;
        }
        sum = warp_sum(sum);
        if (lane == 0) mine[round].mass[warp] = sum;
        if (threadIdx.x == 0) found = -1;
        if (blocks > 1) cluster.sync();
        else __syncthreads();
        const int parts = blocks * kWarps;
        if (warp == 0) {
            // the masses ahead of every part, four parts a lane
            double before = 0.0, m[kMostCluster * kWarps / 32];
#pragma unroll
            for (int k = 0; k < kMostCluster * kWarps / 32; ++k) {
                const int i = lane * (kMostCluster * kWarps / 32) + k;
                m[k] = i < parts ? (double)(blocks > 1 ? cluster.map_shared_rank(&mine[round], i / kWarps) : &mine[round])->mass[i % kWarps] : 0.0;
                before += m[k];
            }
            double incl = before;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double u = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl += u;
            }
            const double total = __shfl_sync(~0u, incl, 31), point = uniform[a.drafts] * total;
            double run = incl - before;
            int here = 0x7FFFFFFF, last = -1;
#pragma unroll
            for (int k = 0; k < kMostCluster * kWarps / 32; ++k) {
                const int i = lane * (kMostCluster * kWarps / 32) + k;
                if (i < parts) ahead_of[i] = run;
                run += m[k];
                if (m[k] > 0.0) {
                    last = i;
                    if (run > point && here == 0x7FFFFFFF) here = i;
                }
            }
            here = warp_min(here), last = __reduce_max_sync(~0u, last);
            if (lane == 0) whole = total, found = here == 0x7FFFFFFF ? last : here;  // (rounding may leave none above)
        }
        __syncthreads();
        chosen = found, want = uniform[a.drafts] * whole;
        if (chosen >= 0 || !refused) break;
        refused = false;  // nothing is left: from p itself
    }
    int64_t *out = a.out + b * (a.drafts + 1);
    float *logprob = a.logprob ? a.logprob + b * (a.drafts + 1) : nullptr;
    auto drawn = [&](int token) {
        out[at] = token;
        if (logprob) logprob[at] = token < 0 ? -INFINITY : log_p(elem<T>::to(lp[token]), token, p);
        a.count[b] = at + 1;
    };
    if (chosen == part) {
        double before = ahead_of[part];
        int token = -1, last = -1;
        for (int v0 = begin; v0 < end && token < 0; v0 += 32 * N) {
            const int v = v0 + lane * N;
            float w[N], s = 0.f;
            if (v < end) weights(v, w);
#pragma unroll
            for (int e = 0; e < N; ++e) s += v < end ? w[e] : 0.f;
            double incl = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double u = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl += u;
            }
            const unsigned above = __ballot_sync(~0u, before + incl > want);
            int mine_last = -1, hit = -1;
            double run = before + incl - s;
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (v < end && w[e] > 0.f) {
                    mine_last = v + e;
                    run += w[e];
                    if (hit < 0 && run > want) hit = v + e;
                }
            if (above) token = __shfl_sync(~0u, hit >= 0 ? hit : mine_last, __ffs(above) - 1);
            last = max(last, __reduce_max_sync(~0u, mine_last));
            before += __shfl_sync(~0u, incl, 31);
        }
        if (lane == 0) drawn(token >= 0 ? token : last);
    } else if (chosen < 0 && part == 0 && lane == 0) {
        drawn(-1);
    }
    if (rank == 0) {
        for (int i = threadIdx.x; i <= a.drafts; i += kThreads)
            if (i != at) {
                out[i] = i < at ? tokens[i] : -1;
                if (logprob) logprob[i] = i < at ? log_of[i] : -INFINITY;
            }
    }
    if (blocks > 1) cluster.sync();  // no block leaves while another reads its masses
}

// How the rows are cut: as many chunks as give all multiprocessors some, of 2,048 to 16,384 logits and a few more.
struct Cut {
    int rows, chunks;
    size_t bytes;
};
Cut cut_for(int sms, int64_t requests, int drafts, bool known, int vocab) {
    Cut c;
    c.rows = known ? 2 * drafts + 1 : drafts + 1;
    int64_t chunks = (4 * (int64_t)sms + requests * c.rows - 1) / (requests * c.rows);
    const int64_t least = (vocab + 17000) / 17001, most = (vocab + 2047) / 2048;
    chunks = chunks < least ? least : chunks > most ? most : chunks;
    c.chunks = (int)chunks;
    c.bytes = sizeof(Stat) * (size_t)requests * c.rows * c.chunks;
    return c;
}

template <typename T> int run(const sim_op_verify_t *a, const Cut &c, cudaStream_t st) {
    constexpr int N = Vec<T>::N;
    const int chunk_len = ((a->vocab + c.chunks - 1) / c.chunks + N - 1) / N * N;
    Stat *stats = (Stat *)a->workspace;
    cudaError_t e = launch_early(k_rows<T>, (unsigned)(a->requests * (int64_t)c.rows * c.chunks), kThreads, 0, 1, st, *a, stats, c.rows, c.chunks, chunk_len);
    if (e != cudaSuccess) return launched("sim_op_verify (rows)", e);
    int blocks = 1;
    while (blocks < kMostCluster && a->vocab > blocks * 4096) blocks *= 2;
    const int step = 32 * N, parts = blocks * kWarps, stretch = ((a->vocab + parts - 1) / parts + step - 1) / step * step;
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
