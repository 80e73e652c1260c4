// quantized_append.cu -- new tokens' rows into the 8-bit block cache (mtsim_ops.h).
#include "eight.cuh"

#include <cmath>

namespace mtop {
namespace {

// A block of threads takes a block of the cache that a request writes: the largest magnitude of
// the rows that come in, the scale that follows, the rows that were there in that
// scale where it has grown, and the new rows.  A warp takes a row at a time.
constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kKeys = 4096;  // rotated elements that are kept in shared memory

// What a block of threads does: request b's rows [r0, r1) of the cache's block `id`, whose row 0 is its token
// `base` and would be row `row0` of the inputs.
struct Work {
    int id, r0, r1;
    int64_t base, row0;
};

// The u-th written block of all requests, looked for by every warp, 32 requests at a time; false: there are fewer.
__device__ __forceinline__ bool find(const sim_op_quantized_append_t &a, int64_t u, Work &w) {
    const int lane = threadIdx.x % 32;
    int64_t seen = 0;
    for (int b0 = 0; b0 < a.requests; b0 += 32) {
        int first = 0, end = 0, units = 0;
        int64_t hi = 0, cached = 0;
        if (b0 + lane < a.requests) {
            const int64_t o0 = a.offsets[b0 + lane], o1 = a.offsets[b0 + lane + 1];
            cached = a.lengths[b0 + lane];
            const int64_t lo = min(max(o0, (int64_t)0), a.tokens);
            hi = min(max(o1, lo), a.tokens);
            // new tokens are [first, end) of the cached ones (indexes below 0 or past the table's end are left out)
            first = (int)max(cached - (hi - lo), (int64_t)0), end = (int)max(min(cached, (int64_t)a.table_blocks * a.block_tokens), (int64_t)0);
            units = end > first ? (end - 1) / a.block_tokens - first / a.block_tokens + 1 : 0;
        }
        int up_to = units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int n = __shfl_up_sync(~0u, up_to, o);
            if (lane >= o) up_to += n;
        }
        const unsigned there = __ballot_sync(~0u, u < seen + up_to);
        if (there) {
            const int who = __ffs(there) - 1;
            const int before = (int)(u - seen) - __shfl_sync(~0u, up_to - units, who);
            first = __shfl_sync(~0u, first, who), end = __shfl_sync(~0u, end, who);
            const int blk = first / a.block_tokens + before;
            w.base = (int64_t)blk * a.block_tokens;
            w.row0 = __shfl_sync(~0u, hi - cached, who) + w.base;
            w.r0 = (int)max(first - w.base, (int64_t)0), w.r1 = (int)min(end - w.base, (int64_t)a.block_tokens);
            w.id = a.table[(int64_t)(b0 + who) * a.table_row + blk];
            return true;
        }
        seen += __shfl_sync(~0u, up_to, 31);
    }
    return false;
}

// The rotated pair of a key that turns by `turns` a position.
template <typename T>
__device__ __forceinline__ float2 turned(const sim_op_quantized_append_t &a, const T *key, int i, unsigned long long turns, int64_t position) {
    const int half = a.rot_dim / 2, i0 = a.layout == SIM_OP_HALF ? i : 2 * i, i1 = a.layout == SIM_OP_HALF ? i + half : 2 * i + 1;
    float c, s;
    angle_cos_sin(turns, position, c, s);
    const float u = elem<T>::to(key[i0]), v = elem<T>::to(key[i1]);
    return make_float2(a.amplitude * (u * c - v * s), a.amplitude * (u * s + v * c));
}
__device__ __forceinline__ float size_of(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
__device__ __forceinline__ float stored(float x, float by) { return fabsf(x) < INFINITY ? x * by : NAN; }
__device__ __forceinline__ uint32_t four_of(const float *f, float by) {
    return pack_e4m3(stored(f[0], by), stored(f[1], by)) | pack_e4m3(stored(f[2], by), stored(f[3], by)) << 16;
}
__device__ __forceinline__ uint32_t four_times(uint32_t w, float by) {
    const float2 x = unpack_e4m3(w & 0xFFFF), y = unpack_e4m3(w >> 16);
    return pack_e4m3(x.x * by, x.y * by) | pack_e4m3(y.x * by, y.y * by) << 16;
}
template <typename T> __device__ __forceinline__ void eight(const T *x, float *f) {
    if (sizeof(T) == 4) ((const Vec<T> *)x)[0].to(f), ((const Vec<T> *)x)[1].to(f + 4);
    else ((const Vec<T> *)x)->to(f);
}

// HOW: an element at a time; rows that are made of whole vectors of 8 elements; the same where a
// warp's rows fit its registers (16-bit rows of up to 512 elements, blocks of up to 16), so that all loads are
// asked for at once and nothing is read again: prompts of 20,000 float16 tokens (32 MB) 13.2 us, else 17.6 (bfloat16 ones, with
// 96 registers instead of 72, in blocks of 12 20.4).
enum { kOnes, kWide, kHeld };
constexpr int kHeldRows = 4, kHeldRank = 512;
template <typename T, int HOW>
__global__ void __launch_bounds__(kThreads) k_quantized_append(const __grid_constant__ sim_op_quantized_append_t a, bool kept) {
    extern __shared__ __align__(16) float keys[];  // rotated, where there is room for a block's
    __shared__ float most[2][kWarps];
    __shared__ unsigned long long per[SIM_OP_MAX_ROT / 2];
    let_next_start();
    after_previous();
    const int half = a.rot_dim / 2, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int i = threadIdx.x; i < half; i += kThreads) per[i] = turns_per_position(a.frequencies[i]);
    Work w;
    if (!find(a, blockIdx.x, w) || w.id < 0 || w.id >= a.blocks) return;
    const T *latent = (const T *)a.latent + w.row0 * a.latent_token;  // of the block's row 0
    const T *key = (const T *)a.key + w.row0 * a.key_token;
    float *scales = a.scales + 2 * (int64_t)w.id;
    const float had0 = scales[0], had1 = scales[1];
    __syncthreads();
    constexpr bool WIDE = HOW != kOnes;
    float m0 = 0.f, m1 = 0.f;
    uint4 held[kHeldRows][2];
    if (HOW == kHeld) {
#pragma unroll
        for (int n = 0; n < kHeldRows; ++n) {
            const int r = w.r0 + warp + n * kWarps;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (r < w.r1 && 8 * (lane + 32 * i) < a.rank) held[n][i] = *(const uint4 *)(latent + r * a.latent_token + 8 * (lane + 32 * i));
        }
    }
    for (int r = w.r0 + warp; r < w.r1; r += kWarps) {
        const T *x = latent + r * a.latent_token, *k = key + r * a.key_token;
        if (HOW == kWide) {
#pragma unroll 2
            for (int i = 8 * lane; i < a.rank; i += 256) {
                float f[8];
                eight(x + i, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) m0 = fmaxf(m0, size_of(f[e]));
            }
        } else if (HOW == kOnes) {
            for (int i = lane; i < a.rank; i += 32) m0 = fmaxf(m0, size_of(elem<T>::to(x[i])));
        }
        for (int i = lane; i < half; i += 32) {
            const float2 v = turned<T>(a, k, i, per[i], w.base + r);
            m1 = fmaxf(m1, fmaxf(size_of(v.x), size_of(v.y)));
            if (kept) {
                float *to = keys + (r - w.r0) * a.rot_dim;
                to[a.layout == SIM_OP_HALF ? i : 2 * i] = v.x, to[a.layout == SIM_OP_HALF ? i + half : 2 * i + 1] = v.y;
            }
        }
    }
    if (HOW == kHeld) {
#pragma unroll
        for (int n = 0; n < kHeldRows; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (w.r0 + warp + n * kWarps < w.r1 && 8 * (lane + 32 * i) < a.rank) {
                    float f[8];
                    eight((const T *)&held[n][i], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) m0 = fmaxf(m0, size_of(f[e]));
                }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m0 = fmaxf(m0, __shfl_xor_sync(~0u, m0, o)), m1 = fmaxf(m1, __shfl_xor_sync(~0u, m1, o));
    if (lane == 0) most[0][warp] = m0, most[1][warp] = m1;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWarps; ++k) m0 = fmaxf(m0, most[0][k]), m1 = fmaxf(m1, most[1][k]);
    float s0 = scale_for(m0), s1 = scale_for(m1);
    uint8_t *rows = (uint8_t *)a.cache + w.id * a.cache_block;
    if (w.r0) {
        const float need0 = s0, need1 = s1;
        s0 = fminf(fmaxf(had0, s0), kLargestScale), s1 = fminf(fmaxf(had1, s1), kLargestScale);
        if (need0 > had0 || need1 > had1)
            for (int r = warp; r < w.r0; r += kWarps) {
                uint8_t *row = rows + r * a.cache_row;
                if (WIDE) {
                    for (int i = 8 * lane; i < a.rank + a.rot_dim; i += 256) {
                        const float by = i < a.rank ? had0 / s0 : had1 / s1;
                        uint2 *at = (uint2 *)(row + i);
                        *at = make_uint2(four_times(at->x, by), four_times(at->y, by));
                    }
                } else {
                    for (int i = lane; i < a.rank + a.rot_dim; i += 32)
                        row[i] = (uint8_t)pack_e4m3(unpack_e4m3(row[i]).x * (i < a.rank ? had0 / s0 : had1 / s1), 0.f);
                }
            }
    }
    const float by0 = 1.f / s0, by1 = 1.f / s1;
    if (HOW == kHeld) {
#pragma unroll
        for (int n = 0; n < kHeldRows; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = w.r0 + warp + n * kWarps, at = 8 * (lane + 32 * i);
                if (r < w.r1 && at < a.rank) {
                    float f[8];
                    eight((const T *)&held[n][i], f);
                    *(uint2 *)(rows + r * a.cache_row + at) = make_uint2(four_of(f, by0), four_of(f + 4, by0));
                }
            }
    }
    for (int r = w.r0 + warp; r < w.r1; r += kWarps) {
        const T *x = latent + r * a.latent_token, *k = key + r * a.key_token;
        uint8_t *row = rows + r * a.cache_row;
        if (HOW == kWide) {
#pragma unroll 2
            for (int i = 8 * lane; i < a.rank; i += 256) {
                float f[8];
                eight(x + i, f);
                *(uint2 *)(row + i) = make_uint2(four_of(f, by0), four_of(f + 4, by0));
            }
        } else if (HOW == kOnes) {
            for (int i = lane; i < a.rank; i += 32) row[i] = (uint8_t)pack_e4m3(stored(elem<T>::to(x[i]), by0), 0.f);
        }
        if (kept) {  // (the warp's own)
            const float *f = keys + (r - w.r0) * a.rot_dim;
            if (WIDE) {
                for (int i = 8 * lane; i < a.rot_dim; i += 256) *(uint2 *)(row + a.rank + i) = make_uint2(four_of(f + i, by1), four_of(f + i + 4, by1));
            } else {
                for (int i = lane; i < a.rot_dim; i += 32) row[a.rank + i] = (uint8_t)pack_e4m3(stored(f[i], by1), 0.f);
            }
        } else {
            for (int i = lane; i < half; i += 32) {
                const float2 v = turned<T>(a, k, i, per[i], w.base + r);
                uint8_t *to = row + a.rank;
                to[a.layout == SIM_OP_HALF ? i : 2 * i] = (uint8_t)pack_e4m3(stored(v.x, by1), 0.f);
                to[a.layout == SIM_OP_HALF ? i + half : 2 * i + 1] = (uint8_t)pack_e4m3(stored(v.y, by1), 0.f);
            }
        }
    }
    if (threadIdx.x == 0) scales[0] = s0, scales[1] = s1;  // (every thread has read them: there were barriers since)
}

template <typename T> int run(const sim_op_quantized_append_t *a, cudaStream_t st) {
    // a request writes its tokens' blocks and one more where they begin inside one
    const int64_t most = a->tokens / a->block_tokens + 2 * (int64_t)a->requests;
    const int n = 16 / (int)sizeof(T);
    const bool wide = a->rank % 8 == 0 && a->rot_dim % 8 == 0 && aligned16(a->latent) && (a->tokens == 1 || a->latent_token % n == 0) &&
                      ((uintptr_t)a->cache & 7) == 0 && (a->blocks == 1 || a->cache_block % 8 == 0) && (a->block_tokens == 1 || a->cache_row % 8 == 0);
    const bool kept = (int64_t)a->block_tokens * a->rot_dim <= kKeys;
    const bool held = wide && sizeof(T) == 2 && a->rank <= kHeldRank && a->block_tokens <= kHeldRows * kWarps;
    return launched("sim_op_quantized_append", launch_early(held ? k_quantized_append<T, sizeof(T) == 2 ? kHeld : kWide> : wide ? k_quantized_append<T, kWide> : k_quantized_append<T, kOnes>, (unsigned)most, kThreads,
                                                            kept ? a->block_tokens * a->rot_dim * 4 : 0, 1, st, *a, kept));
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
    if (a->tokens > INT32_MAX || a->tokens + 2 * (int64_t)a->requests > INT32_MAX) return fail(SIM_ERR_ARG, "a call has fewer than 2^31 tokens");
    if ((int64_t)a->table_blocks * a->block_tokens > INT32_MAX) return fail(SIM_ERR_ARG, "table_blocks * block_tokens must be below 2^31");
    if ((int64_t)a->rank + a->rot_dim > INT32_MAX) return fail(SIM_ERR_ARG, "rank + rot_dim is too large");
    if (a->tokens == 0 || a->requests == 0 || a->blocks == 0 || a->table_blocks == 0) return SIM_OK;
    if (!a->latent || !a->key || !a->frequencies || !a->offsets || !a->table || !a->lengths || !a->cache || !a->scales)
        return fail(SIM_ERR_ARG, "latent, key, frequencies, offsets, table, lengths, cache and scales must not be NULL");
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) return run<__nv_bfloat16>(a, st);
    return a->type == SIM_OP_FP16 ? run<__half>(a, st) : run<float>(a, st);
}
