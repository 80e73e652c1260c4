// quantized_append.cu -- new tokens' rows into the 8-bit block cache (mtsim_ops.h).
#include "eight.cuh"

#include <cmath>

namespace mtop {
namespace {

// A block of threads takes a block of the cache that a request writes: the largest magnitude of
// the rows that come in, the scale that follows, the rows that were there in that
// scale where it has grown, and the new rows.
constexpr int kThreads = 128;

// The rotated pair i of a key.
template <typename T>
__device__ __forceinline__ float2 turned(const sim_op_quantized_append_t &a, const T *key, int i, int position) {
    const int half = a.rot_dim / 2, i0 = a.layout == SIM_OP_HALF ? i : 2 * i, i1 = a.layout == SIM_OP_HALF ? i + half : 2 * i + 1;
    float c, s;
    angle_cos_sin(turns_per_position(a.frequencies[i]), position, c, s);
    const float u = elem<T>::to(key[i0]), v = elem<T>::to(key[i1]);
    return make_float2(a.amplitude * (u * c - v * s), a.amplitude * (u * s + v * c));
}
__device__ __forceinline__ float size_of(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
__device__ __forceinline__ uint8_t byte_of(float x, float by) { return (uint8_t)pack_e4m3(fabsf(x) < INFINITY ? x * by : NAN, 0.f); }

template <typename T>
__global__ void __launch_bounds__(kThreads) k_quantized_append(const __grid_constant__ sim_op_quantized_append_t a) {
    __shared__ float most[2][kThreads / 32];
    let_next_start();
    after_previous();
    const int half = a.rot_dim / 2, width = a.rank + a.rot_dim, lane = threadIdx.x % 32;
    int b = 0;
    int64_t before = 0;  // units (a request's written blocks) of the requests before b
    for (int64_t u = blockIdx.x;; u += gridDim.x) {
        int first = 0, end = 0, n = 0;  // request b's new tokens are [first, end) of its cached ones
        int64_t row0 = 0, units = 0;
        for (; b < a.requests; ++b, before += units) {
            const int64_t lo = min(max((int64_t)a.offsets[b], (int64_t)0), a.tokens), hi = min(max((int64_t)a.offsets[b + 1], lo), a.tokens);
            const int64_t cached = a.lengths[b];
            // (indexes below 0 or past the table's end are left out)
            const int64_t from = max(cached - (hi - lo), (int64_t)0), past = min(cached, (int64_t)a.table_blocks * a.block_tokens);
            row0 = hi - cached;  // the row of token 0
            first = (int)min(from, (int64_t)0x7FFFFFFF), end = (int)max(past, (int64_t)0);
            n = end > first ? end - first : 0;
            units = n ? (end - 1) / a.block_tokens - first / a.block_tokens + 1 : 0;
            if (u < before + units) break;
        }
        if (b == a.requests) return;
        const int blk = first / a.block_tokens + (int)(u - before);
        const int id = a.table[b * a.table_row + blk];
        if (id < 0 || id >= a.blocks) continue;
        const int64_t base = (int64_t)blk * a.block_tokens;
        const int r0 = (int)max(first - base, (int64_t)0), r1 = (int)min(end - base, (int64_t)a.block_tokens);
        const T *latent = (const T *)a.latent + (row0 + base) * a.latent_token;  // of the block's row 0
        const T *key = (const T *)a.key + (row0 + base) * a.key_token;
        float m0 = 0.f, m1 = 0.f;
        for (int64_t k = threadIdx.x; k < (int64_t)(r1 - r0) * a.rank; k += kThreads)
            m0 = fmaxf(m0, size_of(elem<T>::to(latent[(r0 + k / a.rank) * a.latent_token + k % a.rank])));
        for (int64_t k = threadIdx.x; k < (int64_t)(r1 - r0) * half; k += kThreads) {
            const int64_t r = r0 + k / half;
            const float2 v = turned<T>(a, key + r * a.key_token, (int)(k % half), (int)(base + r));
            m1 = fmaxf(m1, fmaxf(size_of(v.x), size_of(v.y)));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) m0 = fmaxf(m0, __shfl_xor_sync(~0u, m0, o)), m1 = fmaxf(m1, __shfl_xor_sync(~0u, m1, o));
        if (lane == 0) most[0][threadIdx.x / 32] = m0, most[1][threadIdx.x / 32] = m1;
        __syncthreads();
        for (int w = 0; w < kThreads / 32; ++w) m0 = fmaxf(m0, most[0][w]), m1 = fmaxf(m1, most[1][w]);
        float *scales = a.scales + 2 * (int64_t)id;
        const float had0 = scales[0], had1 = scales[1];
        float s0 = scale_for(m0), s1 = scale_for(m1);
        uint8_t *rows = (uint8_t *)a.cache + id * a.cache_block;
        if (r0) {
            const float need0 = s0, need1 = s1;
            s0 = fminf(fmaxf(had0, s0), kLargestScale), s1 = fminf(fmaxf(had1, s1), kLargestScale);
            if (need0 > had0 || need1 > had1)
                for (int64_t k = threadIdx.x; k < (int64_t)r0 * width; k += kThreads) {
                    const int j = (int)(k % width);
                    uint8_t *at = rows + k / width * a.cache_row + j;
                    *at = (uint8_t)pack_e4m3(unpack_e4m3(*at).x * (j < a.rank ? had0 / s0 : had1 / s1), 0.f);
                }
        }
        const float by0 = 1.f / s0, by1 = 1.f / s1;
        for (int64_t k = threadIdx.x; k < (int64_t)(r1 - r0) * a.rank; k += kThreads) {
            const int64_t r = r0 + k / a.rank, j = k % a.rank;
            rows[r * a.cache_row + j] = byte_of(elem<T>::to(latent[r * a.latent_token + j]), by0);
        }
        for (int64_t k = threadIdx.x; k < (int64_t)(r1 - r0) * half; k += kThreads) {
            const int64_t r = r0 + k / half;
            const int i = (int)(k % half);
            const float2 v = turned<T>(a, key + r * a.key_token, i, (int)(base + r));
            uint8_t *to = rows + r * a.cache_row + a.rank;
            to[a.layout == SIM_OP_HALF ? i : 2 * i] = byte_of(v.x, by1);
            to[a.layout == SIM_OP_HALF ? i + half : 2 * i + 1] = byte_of(v.y, by1);
        }
        __syncthreads();  // every thread has read the scales, and what others found
        if (threadIdx.x == 0) scales[0] = s0, scales[1] = s1;
    }
}

template <typename T> int run(const sim_op_quantized_append_t *a, int sms, cudaStream_t st) {
    // a request writes its tokens' blocks and one more where they begin inside one
    const int64_t most = a->tokens / a->block_tokens + 2 * (int64_t)a->requests, blocks = 8 * (int64_t)sms;
    return launched("sim_op_quantized_append",
                    launch_early(k_quantized_append<T>, (unsigned)(most < blocks ? most : blocks), kThreads, 0, 1, st, *a));
}

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" int sim_op_quantized_append(const sim_op_quantized_append_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16 && a->type != SIM_OP_FP32) return fail(SIM_ERR_ARG, "unknown element type %d", a->type);
    if (a->layout != SIM_OP_INTERLEAVED && a->layout != SIM_OP_HALF) return fail(SIM_ERR_ARG, "unknown layout %d", a->layout);
    if (a->tokens < 0 || a->requests < 0 || a->blocks < 0 || a->table_blocks < 0) return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a->block_tokens < 1) return fail(SIM_ERR_ARG, "block_tokens must be at least 1");
    if (a->rank < 1) return fail(SIM_ERR_ARG, "rank must be at least 1");
    if (a->rot_dim < 2 || a->rot_dim > SIM_OP_MAX_ROT || a->rot_dim % 2)
        return fail(SIM_ERR_ARG, "rot_dim must be even and in [2, %d]", SIM_OP_MAX_ROT);
    if (!std::isfinite(a->amplitude)) return fail(SIM_ERR_ARG, "amplitude must be finite");
    if (a->tokens > INT32_MAX) return fail(SIM_ERR_ARG, "a call has fewer than 2^31 tokens");
    if ((int64_t)a->table_blocks * a->block_tokens > INT32_MAX) return fail(SIM_ERR_ARG, "table_blocks * block_tokens must be below 2^31");
    if ((int64_t)a->rank + a->rot_dim > INT32_MAX) return fail(SIM_ERR_ARG, "rank + rot_dim is too large");
    if (a->tokens == 0 || a->requests == 0 || a->blocks == 0 || a->table_blocks == 0) return SIM_OK;
    if (!a->latent || !a->key || !a->frequencies || !a->offsets || !a->table || !a->lengths || !a->cache || !a->scales)
        return fail(SIM_ERR_ARG, "latent, key, frequencies, offsets, table, lengths, cache and scales must not be NULL");
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) return run<__nv_bfloat16>(a, sms, st);
    return a->type == SIM_OP_FP16 ? run<__half>(a, sms, st) : run<float>(a, sms, st);
}
