// rotary.cu -- rotary positions, and the write of a token's row into the
// block cache (mtsim_ops.h).
#include "ops.cuh"

#include <initializer_list>

namespace mtop {
namespace {

// Any strides and offsets, an element at a time.
template <typename T>
__global__ void __launch_bounds__(256) k_rotary(sim_op_rotary_t a) {
    __shared__ float2 turn[SIM_OP_MAX_ROT / 2];
    const T *x = (const T *)a.x;
    T *out = (T *)a.out;
    const int half = a.rot_dim / 2;
    let_next_start();
    after_previous();
    for (int64_t n = blockIdx.x; n < a.tokens; n += gridDim.x) {
        const int64_t p = a.positions_64 ? ((const int64_t *)a.positions)[n] : ((const int32_t *)a.positions)[n];
        __syncthreads();
        for (int i = threadIdx.x; i < half; i += blockDim.x) {
            float c, s;
            angle_cos_sin(turns_per_position(a.frequencies[i]), a.inverse ? -p : p, c, s);
            turn[i] = make_float2(c * a.amplitude, s * a.amplitude);
        }
        __syncthreads();
        const T *xr = x + n * a.x_token;
        T *yr = out + n * a.out_token;
        const int rest = a.dim - half;  // a pair counts once, every other element once
        for (int64_t k = threadIdx.x; k < (int64_t)a.heads * rest; k += blockDim.x) {
            const int h = (int)(k / rest), j = (int)(k % rest);
            const T *xh = xr + h * a.x_head;
            T *yh = yr + h * a.out_head;
            if (j < half) {
                const int i0 = a.rot_offset + (a.layout == SIM_OP_HALF ? j : 2 * j);
                const int i1 = a.layout == SIM_OP_HALF ? i0 + half : i0 + 1;
                const float u = elem<T>::to(xh[i0]), v = elem<T>::to(xh[i1]);
                const float2 t = turn[j];
                yh[i0] = elem<T>::from(u * t.x - v * t.y);
                yh[i1] = elem<T>::from(u * t.y + v * t.x);
            } else {
                const int r = j - half, i = r < a.rot_offset ? r : r + a.rot_dim;
                if (x != out) yh[i] = xh[i];
            }
        }
    }
}

// Pairs of a vector (half layout: of two, the first and second elements).
template <typename T, bool HALF> __device__ __forceinline__ void turn_pairs(Vec<T> &a, Vec<T> &b, const float2 *t) {
    constexpr int N = Vec<T>::N;
    float x[N], y[N];
    a.to(x);
    if (HALF) {
        b.to(y);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float r = x[i], s = y[i];
            x[i] = r * t[i].x - s * t[i].y;
            y[i] = r * t[i].y + s * t[i].x;
        }
        b.from(y);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float r = x[i], s = x[i + 1];
            x[i] = r * t[i / 2].x - s * t[i / 2].y;
            x[i + 1] = r * t[i / 2].y + s * t[i / 2].x;
        }
    }
    a.from(x);
}

// The tensors' vectors are aligned and the rotated part is made of whole ones:
// bound by memory.  A block takes a token at a time: its first warps rotate,
// with the token's cosines and sines (computed once, in shared memory) of their
// one vector of a head in registers over all the heads they take; the other
// warps copy the rest of the heads.  (One loop for both made every warp issue
// both: 225 us instead of 128 for 8,192 x 128 heads of 192 with 64 rotated, 805 MB.)
constexpr int kRotaryWarps = 8;

template <typename T, bool HALF>
__global__ void __launch_bounds__(kRotaryWarps * 32) k_rotary_wide(const __grid_constant__ sim_op_rotary_t a, int turn_warps) {
    constexpr int N = Vec<T>::N, P = HALF ? N : N / 2;  // pairs of a thread
    __shared__ float2 turn[SIM_OP_MAX_ROT / 2];
    const int half = a.rot_dim / 2, turned = a.rot_dim / N / (HALF ? 2 : 1), rest = (a.dim - a.rot_dim) / N;
    let_next_start();
    after_previous();
    const bool turns = (int)threadIdx.x < turn_warps * 32;
    const int units = turns ? turned : rest, threads = turns ? turn_warps * 32 : (kRotaryWarps - turn_warps) * 32;
    const int id = turns ? threadIdx.x : threadIdx.x - turn_warps * 32;
    // this thread's vector of a head, the heads it takes: h0, h0 + step, ..
    const int step = units ? threads / units : 0, u = units ? id % units : 0, h0 = step && id / units < step ? id / units : a.heads;
    int at = turns ? a.rot_offset + u * N : u * N;
    if (!turns && at >= a.rot_offset) at += a.rot_dim;
    const int64_t x_step = step * a.x_head, y_step = step * a.out_head;
    unsigned long long per = 0;
    if (threadIdx.x < half) per = turns_per_position(a.frequencies[threadIdx.x]);
    for (int64_t n = blockIdx.x; n < a.tokens; n += gridDim.x) {
        const int64_t p = a.positions_64 ? ((const int64_t *)a.positions)[n] : ((const int32_t *)a.positions)[n];
        const T *x = (const T *)a.x + n * a.x_token + h0 * a.x_head + at;
        T *y = (T *)a.out + n * a.out_token + h0 * a.out_head + at;
        if (!turns) {
            // loads of several heads before their stores: the compiler cannot tell that heads do not overlap
            for (int h = h0; h < a.heads; h += 4 * step) {
                Vec<T> v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k, x += x_step)
                    if (h + k * step < a.heads) v[k] = *(const Vec<T> *)x;
#pragma unroll
                for (int k = 0; k < 4; ++k, y += y_step)
                    if (h + k * step < a.heads) *(Vec<T> *)y = v[k];
            }
            continue;
        }
        named_sync(1, turn_warps * 32);
        for (int i = threadIdx.x; i < half; i += turn_warps * 32) {
            float c, s;
            angle_cos_sin(i == threadIdx.x ? per : turns_per_position(a.frequencies[i]), a.inverse ? -p : p, c, s);
            turn[i] = make_float2(c * a.amplitude, s * a.amplitude);
        }
        named_sync(1, turn_warps * 32);
        float2 t[P];
#pragma unroll
        for (int i = 0; i < P; ++i) t[i] = turn[u * P + i];
        for (int h = h0; h < a.heads; h += 2 * step) {
            Vec<T> v[2], w[2];
#pragma unroll
            for (int k = 0; k < 2; ++k, x += x_step)
                if (h + k * step < a.heads) {
                    v[k] = *(const Vec<T> *)x;
                    if (HALF) w[k] = *(const Vec<T> *)(x + half);
                }
#pragma unroll
            for (int k = 0; k < 2; ++k, y += y_step)
                if (h + k * step < a.heads) {
                    turn_pairs<T, HALF>(v[k], w[k], t);
                    *(Vec<T> *)y = v[k];
                    if (HALF) *(Vec<T> *)(y + half) = w[k];
                }
        }
    }
}

// Any strides and sizes, an element at a time.
template <typename T>
__global__ void __launch_bounds__(128) k_append(sim_op_latent_append_t a) {
    const int half = a.rot_dim / 2;
    let_next_start();
    after_previous();
    for (int64_t n = blockIdx.x; n < a.tokens; n += gridDim.x) {
        const int64_t slot = a.slots[n];
        if (slot < 0 || slot >= a.blocks * a.block_tokens) continue;
        T *row = (T *)a.cache + (slot / a.block_tokens) * a.cache_block + (slot % a.block_tokens) * a.cache_row;
        const T *lat = (const T *)a.latent + n * a.latent_token;
        const T *key = (const T *)a.key + n * a.key_token;
        for (int i = threadIdx.x; i < a.rank; i += blockDim.x) row[i] = lat[i];
        const int64_t p = a.positions_64 ? ((const int64_t *)a.positions)[n] : ((const int32_t *)a.positions)[n];
        for (int i = threadIdx.x; i < half; i += blockDim.x) {
            float c, s;
            angle_cos_sin(turns_per_position(a.frequencies[i]), p, c, s);
            const int i0 = a.layout == SIM_OP_HALF ? i : 2 * i, i1 = a.layout == SIM_OP_HALF ? i + half : 2 * i + 1;
            const float u = elem<T>::to(key[i0]), v = elem<T>::to(key[i1]);
            row[a.rank + i0] = elem<T>::from(a.amplitude * (u * c - v * s));
            row[a.rank + i1] = elem<T>::from(a.amplitude * (u * s + v * c));
        }
    }
}

// The same for whole vectors: a warp takes a token, its lanes the row's
// vectors.  A lane keeps the factor of its first frequency over all its
// tokens, and hands cosines and sines to the lanes that rotate through shared
// memory.  Bound by memory: 20,011 rows of 1,152 bytes to scattered blocks
// (46 MB) take 11.7 us.
constexpr int kAppendWarps = 8;

template <typename T, bool HALF>
__global__ void __launch_bounds__(kAppendWarps * 32, 6) k_append_wide(const __grid_constant__ sim_op_latent_append_t a) {
    constexpr int N = Vec<T>::N, P = HALF ? N : N / 2;
    __shared__ float2 turns[kAppendWarps][SIM_OP_MAX_ROT / 2];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int half = a.rot_dim / 2, turned = a.rot_dim / N / (HALF ? 2 : 1), copied = a.rank / N;
    float2 *turn = turns[warp];
    let_next_start();
    after_previous();
    const unsigned long long per = lane < half ? turns_per_position(a.frequencies[lane]) : 0;
    const int64_t rows = a.blocks * a.block_tokens;
    for (int64_t n = (int64_t)blockIdx.x * kAppendWarps + warp; n < a.tokens; n += (int64_t)gridDim.x * kAppendWarps) {
        // everything that a token needs is loaded at once
        const int64_t slot = a.slots[n];
        const int64_t p = a.positions_64 ? ((const int64_t *)a.positions)[n] : ((const int32_t *)a.positions)[n];
        const T *lat = (const T *)a.latent + n * a.latent_token;
        const T *key = (const T *)a.key + n * a.key_token;
        Vec<T> c0, c1, v, w;
        if (lane < copied) c0 = *(const Vec<T> *)(lat + lane * N);
        if (lane + 32 < copied) c1 = *(const Vec<T> *)(lat + (lane + 32) * N);
        if (lane < turned) {
            v = *(const Vec<T> *)(key + lane * N);
            if (HALF) w = *(const Vec<T> *)(key + half + lane * N);
        }
        for (int i = lane; i < half; i += 32) {
            float c, s;
            angle_cos_sin(i == lane ? per : turns_per_position(a.frequencies[i]), p, c, s);
            turn[i] = make_float2(c * a.amplitude, s * a.amplitude);
        }
        __syncwarp();
        if (slot >= 0 && slot < rows) {
            // (a 64-bit division takes some hundred instructions)
            const int64_t block = rows <= 0xFFFFFFFFll ? (uint32_t)slot / (uint32_t)a.block_tokens : slot / a.block_tokens;
            T *row = (T *)a.cache + block * a.cache_block + (slot - block * a.block_tokens) * a.cache_row;
            if (lane < copied) *(Vec<T> *)(row + lane * N) = c0;
            if (lane + 32 < copied) *(Vec<T> *)(row + (lane + 32) * N) = c1;
            for (int i = lane + 64; i < copied; i += 32) *(Vec<T> *)(row + i * N) = *(const Vec<T> *)(lat + i * N);
            for (int u = lane; u < turned; u += 32) {
                if (u > lane) {
                    v = *(const Vec<T> *)(key + u * N);
                    if (HALF) w = *(const Vec<T> *)(key + half + u * N);
                }
                turn_pairs<T, HALF>(v, w, turn + u * P);
                *(Vec<T> *)(row + a.rank + u * N) = v;
                if (HALF) *(Vec<T> *)(row + a.rank + half + u * N) = w;
            }
        }
        __syncwarp();
    }
}

// Whether every pointer and stride is made of whole vectors of 16 bytes.
bool whole(int n, std::initializer_list<const void *> pointers, std::initializer_list<int64_t> strides) {
    for (const void *p : pointers)
        if (!aligned16(p)) return false;
    for (int64_t s : strides)
        if (s % n) return false;
    return true;
}

template <typename T> int run_rotary(const sim_op_rotary_t *a, cudaStream_t st) {
    constexpr int N = 16 / sizeof(T);
    const bool half = a->layout == SIM_OP_HALF;
    const int turned = a->rot_dim / N / (half ? 2 : 1), rest = (a->dim - a->rot_dim) / N;
    // warps in proportion to the bytes they move; in place nothing is copied
    int turn_warps = a->x == a->out || rest == 0 ? kRotaryWarps : (kRotaryWarps * a->rot_dim + a->dim / 2) / a->dim;
    turn_warps = turn_warps < 1 ? 1 : turn_warps > kRotaryWarps - (rest && a->x != a->out) ? kRotaryWarps - (rest && a->x != a->out) : turn_warps;
    cudaError_t e;
    if (whole(N, {a->x, a->out}, {a->x_token, a->x_head, a->out_token, a->out_head, a->dim, a->rot_offset, half ? a->rot_dim / 2 : a->rot_dim}) &&
        turned <= 32 * turn_warps && (turn_warps == kRotaryWarps || rest <= 32 * (kRotaryWarps - turn_warps))) {
        const unsigned grid = (unsigned)(a->tokens < 16384 ? a->tokens : 16384);
        e = launch_early(half ? k_rotary_wide<T, true> : k_rotary_wide<T, false>, grid, kRotaryWarps * 32, 0, 1, st, *a, turn_warps);
    } else {
        e = launch_early(k_rotary<T>, (unsigned)(a->tokens < (1 << 20) ? a->tokens : (1 << 20)), 256, 0, 1, st, *a);
    }
    return launched("sim_op_rotary", e);
}

template <typename T> int run_append(const sim_op_latent_append_t *a, int sms, cudaStream_t st) {
    constexpr int N = 16 / sizeof(T);
    const bool half = a->layout == SIM_OP_HALF;
    cudaError_t e;
    if (whole(N, {a->latent, a->key, a->cache},
              {a->latent_token, a->key_token, a->cache_block, a->cache_row, a->rank, half ? a->rot_dim / 2 : a->rot_dim})) {
        const int64_t want = (a->tokens + kAppendWarps - 1) / kAppendWarps, most = 6 * (int64_t)sms;
        const unsigned grid = (unsigned)(want < most ? want : most);
        e = launch_early(half ? k_append_wide<T, true> : k_append_wide<T, false>, grid, kAppendWarps * 32, 0, 1, st, *a);
    } else {
        e = launch_early(k_append<T>, (unsigned)(a->tokens < (1 << 20) ? a->tokens : (1 << 20)), 128, 0, 1, st, *a);
    }
    return launched("sim_op_latent_append", e);
}

bool bad_type(int t) { return t != SIM_OP_BF16 && t != SIM_OP_FP16 && t != SIM_OP_FP32; }

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" int sim_op_rotary(const sim_op_rotary_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (bad_type(a->type)) return fail(SIM_ERR_ARG, "unknown element type %d", a->type);
    if (a->layout != SIM_OP_INTERLEAVED && a->layout != SIM_OP_HALF) return fail(SIM_ERR_ARG, "unknown layout %d", a->layout);
    if (a->tokens < 0 || a->heads < 0 || a->dim < 0) return fail(SIM_ERR_ARG, "tokens, heads and dim must not be negative");
    if (a->rot_dim < 2 || a->rot_dim > SIM_OP_MAX_ROT || a->rot_dim % 2)
        return fail(SIM_ERR_ARG, "rot_dim must be even and in [2, %d]", SIM_OP_MAX_ROT);
    if (a->rot_offset < 0 || a->rot_offset > a->dim - a->rot_dim) return fail(SIM_ERR_ARG, "the rotated part does not lie in the head");
    if (a->tokens == 0 || a->heads == 0) return SIM_OK;
    if (!a->x || !a->out || !a->positions || !a->frequencies) return fail(SIM_ERR_ARG, "x, out, positions and frequencies must not be NULL");
    if (a->x == a->out && (a->x_token != a->out_token || a->x_head != a->out_head))
        return fail(SIM_ERR_ARG, "in place, out must have x's strides");
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) return run_rotary<__nv_bfloat16>(a, st);
    return a->type == SIM_OP_FP16 ? run_rotary<__half>(a, st) : run_rotary<float>(a, st);
}

extern "C" int sim_op_latent_append(const sim_op_latent_append_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (bad_type(a->type)) return fail(SIM_ERR_ARG, "unknown element type %d", a->type);
    if (a->layout != SIM_OP_INTERLEAVED && a->layout != SIM_OP_HALF) return fail(SIM_ERR_ARG, "unknown layout %d", a->layout);
    if (a->tokens < 0 || a->blocks < 0) return fail(SIM_ERR_ARG, "tokens and blocks must not be negative");
    if (a->block_tokens < 1) return fail(SIM_ERR_ARG, "block_tokens must be at least 1");
    if (a->rank < 1) return fail(SIM_ERR_ARG, "rank must be at least 1");
    if (a->rot_dim < 2 || a->rot_dim > SIM_OP_MAX_ROT || a->rot_dim % 2)
        return fail(SIM_ERR_ARG, "rot_dim must be even and in [2, %d]", SIM_OP_MAX_ROT);
    if (a->tokens == 0 || a->blocks == 0) return SIM_OK;
    if (!a->latent || !a->key || !a->cache || !a->positions || !a->slots || !a->frequencies)
        return fail(SIM_ERR_ARG, "latent, key, cache, positions, slots and frequencies must not be NULL");
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) return run_append<__nv_bfloat16>(a, sms, st);
    return a->type == SIM_OP_FP16 ? run_append<__half>(a, sms, st) : run_append<float>(a, sms, st);
}
