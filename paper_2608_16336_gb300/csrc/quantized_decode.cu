// quantized_decode.cu -- attention of new tokens over the 8-bit block cache
// of latent vectors (mtsim_ops.h).
#include "eight.cuh"

#include <cmath>

namespace mtop {
namespace {

// A block of threads takes a row (new token x head) of a request, a warp every
// kWarps-th cached token: its lanes hold the query and the warp's sums, with a
// running maximum, and the warps' sums meet at the end.
constexpr int kWarps = 4, kThreads = kWarps * 32, kEach = (SIM_OP_MAX_RANK + SIM_OP_MAX_KEY) / 64;  // pairs of elements of a lane

template <typename T>
__global__ void __launch_bounds__(kThreads) k_quantized_decode(const __grid_constant__ sim_op_quantized_decode_t a) {
    __shared__ float sums[kWarps][SIM_OP_MAX_RANK], tops[kWarps], totals[kWarps];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, width = a.rank + a.key_dim;
    let_next_start();
    after_previous();
    const int64_t row = blockIdx.x, rows = (int64_t)a.new_tokens * a.heads;
    const int64_t b = row / rows, f = row - b * rows, tok = f / a.heads, h = f - tok * a.heads;
    const int64_t cached = min((int64_t)a.lengths[b], (int64_t)a.table_blocks * a.block_tokens);
    const T *q = (const T *)a.q + b * a.q_request + tok * a.q_token + h * a.q_head;
    float2 x[kEach], o[kEach];
    bool odd = false;  // an infinity or NaN in the query
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int j = 2 * (lane + 32 * i);
        x[i] = j < width ? make_float2(elem<T>::to(q[j]), elem<T>::to(q[j + 1])) : make_float2(0.f, 0.f);
        o[i] = make_float2(0.f, 0.f);
        odd |= !(fabsf(x[i].x) < INFINITY) || !(fabsf(x[i].y) < INFINITY);
    }
    odd = __any_sync(~0u, odd);
    float top = -INFINITY, total = 0.f;
    for (int64_t j = warp; j < cached - a.new_tokens + 1 + tok; j += kWarps) {
        const int id = a.table[b * a.table_row + j / a.block_tokens];
        const bool real = id >= 0 && id < a.blocks;
        const float sl = real ? scale_used(a.scales[2 * (int64_t)id]) : 0.f, sk = real ? scale_used(a.scales[2 * (int64_t)id + 1]) : 0.f;
        const uint8_t *c = (const uint8_t *)a.cache + (real ? id * a.cache_block + j % a.block_tokens * a.cache_row : 0);
        float2 v[kEach];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = 2 * (lane + 32 * i);
            const float s = e < a.rank ? sl : sk;
            v[i] = real && e < width ? unpack_e4m3(*(const uint16_t *)(c + e)) : make_float2(0.f, 0.f);
            v[i].x *= s, v[i].y *= s;
            sum += x[i].x * v[i].x + x[i].y * v[i].y;
        }
        const float score = warp_sum(sum) * a.scale;
        const float high = fmaxf(top, score), keep = top == -INFINITY ? 0.f : expf(top - high);
        const float w = score == -INFINITY ? 0.f : expf(score - (high == -INFINITY ? 0.f : high));
        total = total * keep + w;
#pragma unroll
        for (int i = 0; i < kEach; ++i) o[i].x = o[i].x * keep + w * v[i].x, o[i].y = o[i].y * keep + w * v[i].y;
        top = high;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = 2 * (lane + 32 * i);
        if (e < a.rank) sums[warp][e] = o[i].x, sums[warp][e + 1] = o[i].y;
    }
    if (lane == 0) tops[warp] = top, totals[warp] = total;
    __syncthreads();
    float high = -INFINITY, all = 0.f, part[kWarps];
    for (int w = 0; w < kWarps; ++w) high = fmaxf(high, tops[w]);
    for (int w = 0; w < kWarps; ++w) part[w] = tops[w] == -INFINITY ? (totals[w] == 0.f ? 0.f : NAN) : expf(tops[w] - high), all += part[w] * totals[w];
    if (odd && cached - a.new_tokens + 1 + tok > 0) all = NAN;
    T *out = (T *)a.out + b * a.out_request + tok * a.out_token + h * a.out_head;
    for (int e = threadIdx.x; e < a.rank; e += kThreads) {
        float v = 0.f;
        for (int w = 0; w < kWarps; ++w) v += part[w] * sums[w][e];
        out[e] = elem<T>::from(all != 0.f ? v / all : 0.f);
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = all != 0.f ? high + logf(all) : -INFINITY;
}

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" size_t sim_op_quantized_decode_workspace(int32_t requests, int32_t new_tokens, int32_t heads, int32_t rank) {
    (void)requests, (void)new_tokens, (void)heads, (void)rank;
    return 256;
}

extern "C" int sim_op_quantized_decode(const sim_op_quantized_decode_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16) return fail(SIM_ERR_ARG, "element type %d: 16-bit types only", a->type);
    if (a->requests < 0 || a->new_tokens < 0 || a->heads < 0 || a->blocks < 0 || a->table_blocks < 0)
        return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a->rank < 64 || a->rank > SIM_OP_MAX_RANK || a->rank % 64)
        return fail(SIM_ERR_ARG, "rank must be a multiple of 64 in [64, %d]", SIM_OP_MAX_RANK);
    if (a->key_dim < 0 || a->key_dim > SIM_OP_MAX_KEY || a->key_dim % 16)
        return fail(SIM_ERR_ARG, "key_dim must be a multiple of 16 in [0, %d]", SIM_OP_MAX_KEY);
    if (a->block_tokens < 1) return fail(SIM_ERR_ARG, "block_tokens must be at least 1");
    if (!std::isfinite(a->scale)) return fail(SIM_ERR_ARG, "scale must be finite");
    const int64_t rows = (int64_t)a->new_tokens * a->heads;
    if (rows == 0 || a->requests == 0) return SIM_OK;
    if (rows > INT32_MAX || a->requests * rows > INT32_MAX) return fail(SIM_ERR_ARG, "requests * new_tokens * heads must be below 2^31");
    if (!a->q || !a->out || !a->lengths || (!a->table && a->table_blocks) || ((!a->cache || !a->scales) && a->blocks))
        return fail(SIM_ERR_ARG, "q, cache, scales, table, lengths and out must not be NULL");
    if (!aligned16(a->q) || !aligned16(a->cache) || !aligned16(a->out) || !even_stride(a->requests, a->q_request) ||
        !even_stride(a->new_tokens, a->q_token) || !even_stride(a->heads, a->q_head) || !even_stride(a->requests, a->out_request) ||
        !even_stride(a->new_tokens, a->out_token) || !even_stride(a->heads, a->out_head))
        return fail(SIM_ERR_ARG, "q, cache and out must be aligned to 16 bytes, q and out with strides that are multiples of 8 elements");
    if ((a->blocks > 1 && a->cache_block % 16) || (a->block_tokens > 1 && a->cache_row % 16))
        return fail(SIM_ERR_ARG, "the cache's strides must be multiples of 16 elements");
    // the cache is one line of rows to the copies: a block must begin on one (blocks of one row are the rows)
    const int64_t cache_row = a->block_tokens > 1 ? a->cache_row : a->blocks > 1 && a->cache_block ? a->cache_block : a->rank + a->key_dim;
    if (cache_row < a->rank + a->key_dim || (a->blocks > 1 && (a->cache_block < 0 || a->cache_block % cache_row)))
        return fail(SIM_ERR_ARG, "cache_block must be a multiple of cache_row, which must hold a row");
    const int64_t ratio = a->blocks > 1 ? a->cache_block / cache_row : a->block_tokens, cache_rows = a->blocks ? (a->blocks - 1) * ratio + a->block_tokens : 0;
    if (cache_rows > INT32_MAX - 1 || ratio > INT32_MAX) return fail(SIM_ERR_ARG, "the cache must span fewer than 2^31 - 1 rows");
    const int64_t most = (int64_t)a->table_blocks * a->block_tokens;
    if (most > INT32_MAX - 65536) return fail(SIM_ERR_ARG, "table_blocks * block_tokens must be below 2^31 - 2^16");
    if (a->requests * (most / 32 + 1) > INT32_MAX) return fail(SIM_ERR_ARG, "requests * table_blocks * block_tokens is too large");
    if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < 256)
        return fail(SIM_ERR_ARG, "a workspace aligned to 256 bytes is needed");
    sim_op_quantized_decode_t k = *a;
    k.cache_row = cache_row;
    if (a->blocks <= 1) k.cache_block = 0;
    const cudaStream_t st = (cudaStream_t)stream;
    const unsigned grid = (unsigned)(a->requests * rows);
    return launched("sim_op_quantized_decode", a->type == SIM_OP_BF16 ? launch_early(k_quantized_decode<__nv_bfloat16>, grid, kThreads, 0, 1, st, k)
                                                                      : launch_early(k_quantized_decode<__half>, grid, kThreads, 0, 1, st, k));
}
