// sample.cu -- one token per row of logits (mtsim_ops.h).
#include "ops.cuh"

#include <cmath>

namespace mtop {
namespace {

constexpr int kThreads = 1024;
typedef unsigned long long u64;

// Weights are whole numbers of 2^-40: their sums are exact, so neither the
// order of the additions nor the split over threads changes a result.
constexpr float kUnit = 1099511627776.f;

// Order-preserving whole number of a logit; NaN ranks with -infinity, -0 with 0.
__device__ __forceinline__ uint32_t key_of(float v) {
    if (!(v > -INFINITY)) v = -INFINITY;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

struct Row {
    float top, per;  // the largest logit, log2(e) / temperature
    float floor_w;   // min_p
    __device__ float weight(float v) const {
        if (top == INFINITY) return v == INFINITY ? 1.f : 0.f;
        return exp2f((v - top) * per);
    }
    __device__ u64 units(float v) const { return __float2ull_rn(weight(v) * kUnit); }
};

template <typename V>
__device__ V block_sum(V v, V *tmp) {
    __syncthreads();
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (threadIdx.x % 32 == 0) tmp[threadIdx.x / 32] = v;
    __syncthreads();
    V s = 0;
    for (int w = 0; w < kThreads / 32; ++w) s += tmp[w];
    return s;
}

// One block per row; thresholds by bisection over the keys.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample(sim_op_sample_t a) {
    __shared__ u64 tmp[32];
    __shared__ uint32_t tmp32[32];
    __shared__ u64 before_of[33];
    __shared__ int found;
    const int row = blockIdx.x, v = a.vocab;
    const T *x = (const T *)a.logits + row * a.logits_row;
    auto at = [&](int i) { return elem<T>::to(x[i]); };
    uint32_t best = 0;
    for (int i = threadIdx.x; i < v; i += kThreads) best = max(best, key_of(at(i)));
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(~0u, best, o));
    if (threadIdx.x % 32 == 0) tmp32[threadIdx.x / 32] = best;
    __syncthreads();
    for (int w = 0; w < 32; ++w) best = max(best, tmp32[w]);
    Row r;
    r.top = value_of(best);
    const float t = a.temperature ? a.temperature[row] : 1.f;
    const bool greedy = !(t > 0);
    r.per = 1.4426950408889634f / t;
    r.floor_w = a.min_p ? fminf(a.min_p[row], 1.f) : 0.f;  // the largest logit always stays
    if (r.top == -INFINITY) {
        if (threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    // kept: keys above `bound`, and the first `ties` (by index) of those equal to it
    uint32_t bound = 0;
    int ties = v;
    if (greedy) bound = best, ties = 1;
    const int k = a.top_k ? a.top_k[row] : 0;
    if (!greedy && k > 0 && k < v) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = bound | 1u << bit;
            uint32_t n = 0;
            for (int i = threadIdx.x; i < v; i += kThreads) n += key_of(at(i)) >= c;
            if (block_sum(n, tmp32) >= (uint32_t)k) bound = c;
        }
        uint32_t n = 0;
        for (int i = threadIdx.x; i < v; i += kThreads) n += key_of(at(i)) > bound;
        ties = k - (int)block_sum(n, tmp32);
    }
    const float p = a.top_p ? a.top_p[row] : 1.f;
    if (!greedy && p < 1.f) {
        u64 m = 0;
        for (int i = threadIdx.x; i < v; i += kThreads) m += key_of(at(i)) > bound ? r.units(at(i)) : 0;
        const u64 each = r.units(value_of(bound));
        u64 all = block_sum(m, tmp);
        if (bound) all += (u64)ties * each;
        else {  // every token counts
            m = 0;
            for (int i = threadIdx.x; i < v; i += kThreads) m += r.units(at(i));
            all = block_sum(m, tmp);
        }
        u64 want = (u64)ceil((double)(p > 0 ? p : 0.f) * (double)all);
        if (want < 1) want = 1;
        uint32_t b2 = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = b2 | 1u << bit;
            m = 0;
            for (int i = threadIdx.x; i < v; i += kThreads) m += key_of(at(i)) >= c ? r.units(at(i)) : 0;
            if (block_sum(m, tmp) >= want) b2 = c;
        }
        if (b2 >= bound) {
            m = 0;
            for (int i = threadIdx.x; i < v; i += kThreads) m += key_of(at(i)) > b2 ? r.units(at(i)) : 0;
            const u64 over = block_sum(m, tmp), unit = r.units(value_of(b2));
            const u64 need = unit && want > over ? (want - over + unit - 1) / unit : 1;
            if (b2 > bound) bound = b2, ties = v;
            if (need < (u64)ties) ties = (int)need;
        }
    }
    // the draw, in vocabulary order: a warp owns a contiguous part of each tile
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    u64 total = 0, target = 0, seen = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int tied = 0;
        if (threadIdx.x == 0) found = v;
        for (int i0 = 0; i0 < v; i0 += kThreads) {
            const int i = i0 + threadIdx.x;
            const float xv = i < v ? at(i) : -INFINITY;
            const uint32_t key = key_of(xv);
            const bool tie = i < v && key == bound;
            const uint32_t votes = __ballot_sync(~0u, tie);
            __syncthreads();
            if (lane == 0) tmp32[warp] = __popc(votes);
            __syncthreads();
            int rank = tied + __popc(votes & ((1u << lane) - 1));
            for (int w = 0; w < 32; ++w) {
                if (w < warp) rank += tmp32[w];
                tied += tmp32[w];
            }
            const bool kept = i < v && (key > bound || (tie && rank < ties)) && (greedy || r.weight(xv) >= r.floor_w);
            const u64 w = kept ? (greedy ? 1 : r.units(xv)) : 0;
            u64 incl = w;
            for (int o = 1; o < 32; o <<= 1) {
                const u64 u = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl += u;
            }
            if (lane == 31) before_of[warp] = incl;
            __syncthreads();
            u64 base = seen;
            for (int q = 0; q < 32; ++q) {
                if (q < warp) base += before_of[q];
                seen += before_of[q];
            }
            if (pass == 1 && w && base + incl > target && base + incl - w <= target) found = i;
        }
        if (pass == 0) {
            total = seen;
            const float u = a.uniform[row];
            target = (u64)((double)(u > 0 ? u : 0.f) * (double)total);
            if (target >= total) target = total - 1;
            seen = 0;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.token[row] = found < v ? found : -1;
        if (a.logprob) {
            const float share = greedy || found >= v ? 1.f : (float)((double)total / (double)kUnit);
            const float l = found < v ? at(found) : 0.f;
            a.logprob[row] = greedy ? 0.f : (r.top == INFINITY ? 0.f : (l - r.top) / t) - logf(share);
        }
    }
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
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) k_sample<__nv_bfloat16><<<a->rows, kThreads, 0, st>>>(*a);
    else if (a->type == SIM_OP_FP16) k_sample<__half><<<a->rows, kThreads, 0, st>>>(*a);
    else k_sample<float><<<a->rows, kThreads, 0, st>>>(*a);
    return launched("sim_op_sample");
}
