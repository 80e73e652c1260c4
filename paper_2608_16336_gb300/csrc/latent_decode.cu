// latent_decode.cu -- attention of new tokens over the block cache of latent
// vectors (mtsim_ops.h).
#include "ops.cuh"

#include <cmath>

namespace mtop {
namespace {

constexpr int kWarps = 4;

// One block per (request, new token, head); a warp takes every fourth cached
// row with a softmax of its own, joined at the end.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) k_decode(sim_op_latent_decode_t a) {
    __shared__ float part[kWarps][SIM_OP_MAX_RANK];
    __shared__ float top_of[kWarps], sum_of[kWarps];
    const int h = blockIdx.x % a.heads, t = blockIdx.x / a.heads % a.new_tokens, b = blockIdx.x / a.heads / a.new_tokens;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int width = a.rank + a.key_dim;
    const T *q = (const T *)a.q + b * a.q_request + t * a.q_token + h * a.q_head;
    const int64_t most = (int64_t)a.table_blocks * a.block_tokens;
    const int64_t len = min((int64_t)a.lengths[b], most), sees = min(len, len - a.new_tokens + 1 + t);
    float qv[18], acc[16], top = -INFINITY, sum = 0;
#pragma unroll
    for (int i = 0; i < 18; ++i) qv[i] = lane + 32 * i < width ? elem<T>::to(q[lane + 32 * i]) : 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0;
    for (int64_t j = warp; j < sees; j += kWarps) {
        const int32_t blk = a.table[b * a.table_row + j / a.block_tokens];
        const bool real = blk >= 0 && blk < a.blocks;
        const T *c = (const T *)a.cache + (real ? blk * a.cache_block + (j % a.block_tokens) * a.cache_row : 0);
        float cv[18], s = 0;
#pragma unroll
        for (int i = 0; i < 18; ++i) {
            cv[i] = real && lane + 32 * i < width ? elem<T>::to(c[lane + 32 * i]) : 0.f;
            s += qv[i] * cv[i];
        }
        s = warp_sum(s) * a.scale;
        const float t2 = fmaxf(top, s), keep = top == -INFINITY ? 0.f : expf(top - t2);
        const float e1 = expf(s - t2), w = elem<T>::to(elem<T>::from(e1));
        top = t2;
        sum = sum * keep + e1;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = acc[i] * keep + w * cv[i];
    }
    if (lane == 0) top_of[warp] = top, sum_of[warp] = sum;
#pragma unroll
    for (int i = 0; i < 16; ++i) part[warp][lane + 32 * i] = acc[i];
    __syncthreads();
    float m = -INFINITY, total = 0, f[kWarps];
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, top_of[w]);
    for (int w = 0; w < kWarps; ++w) {
        f[w] = top_of[w] == -INFINITY ? 0.f : expf(top_of[w] - m);
        total += f[w] * sum_of[w];
    }
    T *out = (T *)a.out + b * a.out_request + t * a.out_token + h * a.out_head;
    for (int i = threadIdx.x; i < a.rank; i += blockDim.x) {
        float v = 0;
        for (int w = 0; w < kWarps; ++w) v += f[w] * part[w][i];
        out[i] = elem<T>::from(total > 0 ? v / total : 0.f);
    }
    if (a.lse && threadIdx.x == 0) a.lse[blockIdx.x] = total > 0 ? m + logf(total) : -INFINITY;
}

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" size_t sim_op_latent_decode_workspace(int32_t, int32_t, int32_t, int32_t) { return 256; }

extern "C" int sim_op_latent_decode(const sim_op_latent_decode_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16) return fail(SIM_ERR_ARG, "element type %d: 16-bit types only", a->type);
    if (a->requests < 0 || a->new_tokens < 0 || a->heads < 0 || a->blocks < 0 || a->table_blocks < 0)
        return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a->rank < 64 || a->rank > SIM_OP_MAX_RANK || a->rank % 64)
        return fail(SIM_ERR_ARG, "rank must be a multiple of 64 in [64, %d]", SIM_OP_MAX_RANK);
    if (a->key_dim < 0 || a->key_dim > SIM_OP_MAX_KEY || a->key_dim % 8)
        return fail(SIM_ERR_ARG, "key_dim must be a multiple of 8 in [0, %d]", SIM_OP_MAX_KEY);
    if (a->block_tokens < 1) return fail(SIM_ERR_ARG, "block_tokens must be at least 1");
    if (!std::isfinite(a->scale)) return fail(SIM_ERR_ARG, "scale must be finite");
    const int64_t rows = (int64_t)a->requests * a->new_tokens * a->heads;
    if (rows == 0) return SIM_OK;
    if (rows > INT32_MAX) return fail(SIM_ERR_ARG, "requests * new_tokens * heads must be below 2^31");
    if (!a->q || !a->out || !a->lengths || (!a->table && a->table_blocks) || (!a->cache && a->blocks))
        return fail(SIM_ERR_ARG, "q, cache, table, lengths and out must not be NULL");
    if (!aligned16(a->q) || !aligned16(a->cache) || !aligned16(a->out) || a->q_request % 8 || a->q_token % 8 || a->q_head % 8 ||
        a->cache_block % 8 || a->cache_row % 8 || a->out_request % 8 || a->out_token % 8 || a->out_head % 8)
        return fail(SIM_ERR_ARG, "q, cache and out must be aligned to 16 bytes, with strides that are multiples of 8 elements");
    if (!a->workspace || a->workspace_bytes < sim_op_latent_decode_workspace(a->requests, a->new_tokens, a->heads, a->rank))
        return fail(SIM_ERR_ARG, "the workspace is too small");
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) k_decode<__nv_bfloat16><<<(unsigned)rows, kWarps * 32, 0, st>>>(*a);
    else k_decode<__half><<<(unsigned)rows, kWarps * 32, 0, st>>>(*a);
    return launched("sim_op_latent_decode");
}
