// verify.cu -- which drafted tokens the target's probabilities keep, and the
// token that follows them (mtsim_ops.h).
#include "ops.cuh"

namespace mtop {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

// log2(e) / t in two floats: (l - m) * (hi + lo) is the binary logarithm of a weight.
struct Rate {
    float hi, lo;
    bool greedy;
    __device__ explicit Rate(float t) {
        greedy = !(t > 0.f);
        const double r = greedy ? 0.0 : 1.4426950408889634 / (double)t;
        hi = (float)r, lo = hi < INFINITY ? (float)(r - (double)hi) : 0.f;
    }
};

// A row of logits with its largest one m, the sum of the weights 2^(rate (l - m)), and the
// lowest index of m (greedy rows: all of the weight).
struct Row {
    float m;
    double sum;
    int first;
};

// A weight to about 2^-22 of itself: the exponent's rounding (2^-24 of up to
// 100) is kept apart and multiplied in.
__device__ __forceinline__ float weight_of(float l, int v, const Row &r, const Rate &c) {
    if (c.greedy) return v == r.first ? 1.f : 0.f;
    if (!(l > -INFINITY)) return 0.f;  // (or NaN)
    if (r.m == INFINITY) return l == INFINITY ? 1.f : 0.f;
    const float d = __fsub_rn(l, r.m), b = __fsub_rn(d, l), off = __fsub_rn(__fsub_rn(l, __fsub_rn(d, b)), __fadd_rn(r.m, b));  // d + off = l - m
    const float y = __fmul_rn(d, c.hi);
    if (!(y > -126.f)) return 0.f;
    const float e = fmaf(d, c.hi, -y) + fmaf(d, c.lo, off * c.hi);
    float p;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(y));
    return fmaf(p, e * 0.6931471805599453f, p);
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

template <typename T> __device__ Row look(const T *x, int vocab, const Rate &c) {
    __shared__ float tops[kWarps];
    __shared__ int firsts[kWarps];
    __shared__ double sums[kWarps];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    Row r = {-INFINITY, 0.0, 0x7FFFFFFF};
    for (int v = threadIdx.x; v < vocab; v += kThreads) {
        const float l = elem<T>::to(x[v]);
        if (l > r.m) r.m = l, r.first = v;
    }
    auto meet = [&](float m, int first) {
        if (m > r.m || (m == r.m && first < r.first)) r.m = m, r.first = first;
    };
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m = __shfl_xor_sync(~0u, r.m, o);
        const int first = __shfl_xor_sync(~0u, r.first, o);
        meet(m, first);
    }
    __syncthreads();
    if (lane == 0) tops[warp] = r.m, firsts[warp] = r.first;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) meet(tops[w], firsts[w]);
    float sum = 0.f;
    for (int v = threadIdx.x; v < vocab; v += kThreads) sum += weight_of(elem<T>::to(x[v]), v, r, c);
    const double all = warp_sum((double)sum);
    if (lane == 0) sums[warp] = all;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) r.sum += sums[w];
    return r;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_verify(const __grid_constant__ sim_op_verify_t a) {
    __shared__ double sums[kWarps + 1];
    __shared__ int found;
    let_next_start();
    after_previous();
    const int64_t b = blockIdx.x;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int drafted = a.drafted ? min(max(a.drafted[b], 0), a.drafts) : a.drafts;
    const Rate rate(a.temperature ? a.temperature[b] : 1.f);
    const T *target = (const T *)a.target + b * a.target_request, *draft = a.draft ? (const T *)a.draft + b * a.draft_request : nullptr;
    const int64_t *tokens = a.tokens + b * a.drafts;
    const float *uniform = a.uniform + b * (a.drafts + 1);
    int64_t *out = a.out + b * (a.drafts + 1);
    float *logprob = a.logprob ? a.logprob + b * (a.drafts + 1) : nullptr;
    auto log_of = [&](float l, int v, const Row &p) {
        const float w = weight_of(l, v, p, rate);
        if (!(w > 0.f)) return -INFINITY;
        if (rate.greedy) return 0.f;
        return (float)(p.m == INFINITY ? -log(p.sum) : ((double)l - p.m) * ((double)rate.hi + rate.lo) * 0.6931471805599453 - log(p.sum));
    };
    int at = 0;
    Row p, q = {0.f, 1.0, 0};
    bool refused = false;
    for (;; ++at) {
        p = look<T>(target + at * a.target_row, a.vocab, rate);
        if (at == drafted) break;
        const int64_t x = tokens[at];
        const bool real = x >= 0 && x < a.vocab;
        if (draft) q = look<T>(draft + at * a.draft_row, a.vocab, rate);
        const float l = real ? elem<T>::to(target[at * a.target_row + x]) : -INFINITY;
        const double px = real && p.sum > 0.0 ? weight_of(l, (int)x, p, rate) / p.sum : 0.0;
        const double qx = !real ? 0.0 : !draft ? 1.0 : q.sum > 0.0 ? weight_of(elem<T>::to(draft[at * a.draft_row + x]), (int)x, q, rate) / q.sum : 0.0;
        if (!(uniform[at] * qx < px)) {
            refused = true;
            break;
        }
        if (threadIdx.x == 0) {
            out[at] = x;
            if (logprob) logprob[at] = log_of(l, (int)x, p);
        }
    }
    // the draw, in pieces of kThreads tokens
    const T *lp = target + at * a.target_row, *lq = draft && refused ? draft + at * a.draft_row : nullptr;
    const int64_t x = refused ? tokens[at] : -1;
    const float by_p = p.sum > 0.0 ? (float)(1.0 / p.sum) : 0.f, by_q = q.sum > 0.0 ? (float)(1.0 / q.sum) : 0.f;
    auto rest = [&](int v) {
        // (two roundings and not one fused step: equal probabilities leave nothing)
        const float w = __fmul_rn(weight_of(elem<T>::to(lp[v]), v, p, rate), by_p);
        if (!refused) return w;
        if (!lq) return v == x ? fmaxf(__fsub_rn(w, 1.f), 0.f) : w;
        return fmaxf(__fsub_rn(w, __fmul_rn(weight_of(elem<T>::to(lq[v]), v, q, rate), by_q)), 0.f);
    };
    double total = 0.0;
    for (int round = 0; round < 2; ++round) {
        double sum = 0.0;
        for (int v = threadIdx.x; v < a.vocab; v += kThreads) sum += rest(v);
        sum = warp_sum(sum);
        __syncthreads();
        if (lane == 0) sums[warp] = sum;
        __syncthreads();
        total = 0.0;
        for (int w = 0; w < kWarps; ++w) total += sums[w];
        if (total > 0.0 || !refused) break;
        refused = false;  // nothing is left: from p itself
    }
    int token = -1;
    if (total > 0.0) {
        const double want = uniform[a.drafts] * total;
        double before = 0.0;
        int last = -1;  // the last token with weight, should rounding leave none above
        if (threadIdx.x == 0) found = 0x7FFFFFFF;
        for (int v0 = 0; v0 < a.vocab && token < 0; v0 += kThreads) {
            const int v = v0 + threadIdx.x;
            const float w = v < a.vocab ? rest(v) : 0.f;
            double incl = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double u = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl += u;
            }
            __syncthreads();
            if (lane == 31) sums[warp] = incl;
            __syncthreads();
            double ahead = before;
            for (int k = 0; k < warp; ++k) ahead += sums[k];
            if (w > 0.f) {
                last = v;
                if (ahead + incl > want) atomicMin(&found, v);
            }
            for (int k = 0; k < kWarps; ++k) before += sums[k];
            __syncthreads();
            if (found != 0x7FFFFFFF) token = found;
        }
        if (token < 0) {
            __syncthreads();
            if (threadIdx.x == 0) found = -1;
            __syncthreads();
            atomicMax(&found, last);
            __syncthreads();
            token = found;
        }
    }
    if (threadIdx.x == 0) {
        out[at] = token;
        if (logprob) logprob[at] = token < 0 ? -INFINITY : log_of(elem<T>::to(lp[token]), token, p);
        a.count[b] = at + 1;
    }
    for (int i = at + 1 + threadIdx.x; i <= a.drafts; i += kThreads) {
        out[i] = -1;
        if (logprob) logprob[i] = -INFINITY;
    }
}

}  // namespace
}  // namespace mtop

using namespace mtop;

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
    const cudaStream_t st = (cudaStream_t)stream;
    const unsigned grid = (unsigned)a->requests;
    cudaError_t e;
    if (a->type == SIM_OP_BF16) e = launch_early(k_verify<__nv_bfloat16>, grid, kThreads, 0, 1, st, *a);
    else if (a->type == SIM_OP_FP16) e = launch_early(k_verify<__half>, grid, kThreads, 0, 1, st, *a);
    else e = launch_early(k_verify<float>, grid, kThreads, 0, 1, st, *a);
    return launched("sim_op_verify", e);
}
