// rotary.cu -- rotary positions, and the write of a token's row into the
// block cache (mtsim_ops.h).
#include "ops.cuh"

#include <initializer_list>

namespace mtop {
namespace {

// Any strides and offsets, an element at a time.  Bound by instructions, a 64-bit
// division an element among them: 8,192 tokens x 128 heads of 192 an element off a
// vector's place take 451 us (whole vectors 121), 1,000 x 16 heads 10.6 (6.0).
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
// bound by memory.  A block takes a group of tokens at a time, computes all their
// cosines and sines in shared memory, and its threads take vectors (pairs of them
// in the half layout) of any token and head: first all that rotate, then all that are copied,
// so that no warp does both.  8,192 tokens x 128 heads of 192 with 64 rotated
// (805 MB) take 122 to 125 us, 6.5 TB/s; 13,850 x 12 heads of 104 (69 MB) 15 us; 11,407
// tokens of 32 floats 6 us.
constexpr int kGroupThreads = 256, kGroupBlocks = 4, kGroupTurns = 1024, kGroupVectors = 2048;

// u / d for u, d < 2^16 (d = 0: there is no u)
struct Divider {
    uint32_t d, m;
    __host__ explicit Divider(uint32_t by) : d(by), m(by > 1 ? (uint32_t)(((1ull << 32) + by - 1) / by) : 0) {}
    __device__ __forceinline__ uint32_t operator()(uint32_t u) const { return d == 1 ? u : __umulhi(u, m); }
};
struct Group {
    int tokens;
    Divider turned_token, turned_head, rest_token, rest_head;  // vectors of a token and of a head
};

template <typename T, bool HALF>
__global__ void __launch_bounds__(kGroupThreads, kGroupBlocks) k_rotary_wide(const __grid_constant__ sim_op_rotary_t a, const __grid_constant__ Group g) {
    constexpr int N = Vec<T>::N, P = HALF ? N : N / 2;
    __shared__ __align__(16) float2 turn[kGroupTurns];
    __shared__ unsigned long long per[SIM_OP_MAX_ROT / 2];
    const int half = a.rot_dim / 2;
    let_next_start();
    after_previous();
    if (threadIdx.x < half) per[threadIdx.x] = turns_per_position(a.frequencies[threadIdx.x]);
    for (int64_t n0 = (int64_t)blockIdx.x * g.tokens; n0 < a.tokens; n0 += (int64_t)gridDim.x * g.tokens) {
        const uint32_t here = (uint32_t)min((int64_t)g.tokens, a.tokens - n0);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < here * half; i += kGroupThreads) {
            const uint32_t tok = i / half;
            const int64_t n = n0 + tok, p = a.positions_64 ? ((const int64_t *)a.positions)[n] : ((const int32_t *)a.positions)[n];
            float c, s;
            angle_cos_sin(per[i - tok * half], a.inverse ? -p : p, c, s);
            turn[i] = make_float2(c * a.amplitude, s * a.amplitude);
        }
        __syncthreads();
        const T *x = (const T *)a.x + n0 * a.x_token;
        T *y = (T *)a.out + n0 * a.out_token;
        // loads of two vectors (or pairs of vectors) before their stores
        const uint32_t turned = here * g.turned_token.d, rest = a.x == a.out ? 0 : here * g.rest_token.d;
        for (uint32_t u0 = threadIdx.x; u0 < turned; u0 += 2 * kGroupThreads) {
            Vec<T> v[2], w[2];
            int64_t to[2];
            uint32_t t_at[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t u = u0 + k * kGroupThreads;
                if (u < turned) {
                    const uint32_t tok = g.turned_token(u), r = u - tok * g.turned_token.d, h = g.turned_head(r), j = r - h * g.turned_head.d;
                    const T *from = x + tok * a.x_token + h * a.x_head + a.rot_offset + j * N;
                    v[k] = *(const Vec<T> *)from;
                    if (HALF) w[k] = *(const Vec<T> *)(from + half);
                    to[k] = tok * a.out_token + h * a.out_head + a.rot_offset + j * N, t_at[k] = tok * half + j * P;
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (u0 + k * kGroupThreads < turned) {
                    turn_pairs<T, HALF>(v[k], w[k], turn + t_at[k]);
                    *(Vec<T> *)(y + to[k]) = v[k];
                    if (HALF) *(Vec<T> *)(y + to[k] + half) = w[k];
                }
        }
        for (uint32_t u0 = threadIdx.x; u0 < rest; u0 += 4 * kGroupThreads) {
            Vec<T> v[4];
            int64_t to[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t u = u0 + k * kGroupThreads;
                if (u < rest) {
                    const uint32_t tok = g.rest_token(u), r = u - tok * g.rest_token.d, h = g.rest_head(r);
                    int at = (int)(r - h * g.rest_head.d) * N;
                    if (at >= a.rot_offset) at += a.rot_dim;
                    v[k] = *(const Vec<T> *)(x + tok * a.x_token + h * a.x_head + at);
                    to[k] = tok * a.out_token + h * a.out_head + at;
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (u0 + k * kGroupThreads < rest) *(Vec<T> *)(y + to[k]) = v[k];
        }
    }
}

// Any strides and sizes, an element at a time: 20,011 rows an element off a vector's
// place 22.6 us (whole vectors 14.5; the host's slices included).
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

template <typename T> int run_rotary(const sim_op_rotary_t *a, int sms, cudaStream_t st) {
    constexpr int N = 16 / sizeof(T);
    const bool half = a->layout == SIM_OP_HALF;
    const int turned = a->rot_dim / N / (half ? 2 : 1), rest = (a->dim - a->rot_dim) / N;
    const int64_t most = (int64_t)a->heads * (turned > rest ? turned : rest);  // vectors of a token
    cudaError_t e;
    if (most < 65536 && whole(N, {a->x, a->out}, {a->x_token, a->x_head, a->out_token, a->out_head, a->dim, a->rot_offset, half ? a->rot_dim / 2 : a->rot_dim})) {
        // As many tokens as give a thread eight vectors, while every block has a group:
        // 16,384 tokens, 24 heads of 192 50 to 53 us with 4 to 8 tokens (one 77.5), 12,000 x 8
        // heads 12 us with 12 (one 30); 8,192 x 128 heads 122 us with one (two 131).
        int64_t group = a->tokens / (kGroupBlocks * (int64_t)sms);
        if (group > kGroupVectors / most) group = kGroupVectors / most;
        if (group > kGroupTurns / (a->rot_dim / 2)) group = kGroupTurns / (a->rot_dim / 2);
        if (group < 1) group = 1;
        const Group g = {(int)group, Divider(a->heads * turned), Divider(turned), Divider(a->heads * rest), Divider(rest)};
        const int64_t groups = (a->tokens + group - 1) / group, blocks = kGroupBlocks * (int64_t)sms;
        const unsigned grid = (unsigned)(groups < blocks ? groups : blocks);
        e = launch_early(half ? k_rotary_wide<T, true> : k_rotary_wide<T, false>, grid, kGroupThreads, 0, 1, st, *a, g);
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
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) return run_rotary<__nv_bfloat16>(a, sms, st);
    return a->type == SIM_OP_FP16 ? run_rotary<__half>(a, sms, st) : run_rotary<float>(a, sms, st);
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
