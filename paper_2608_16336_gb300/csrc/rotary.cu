// rotary.cu -- rotary positions, and the write of a token's row into the
// block cache (mtsim_ops.h).
#include "ops.cuh"

namespace mtop {
namespace {

template <typename T>
__global__ void __launch_bounds__(256) k_rotary(sim_op_rotary_t a) {
    __shared__ float2 turn[SIM_OP_MAX_ROT / 2];
    const T *x = (const T *)a.x;
    T *out = (T *)a.out;
    const int half = a.rot_dim / 2;
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

template <typename T>
__global__ void __launch_bounds__(128) k_append(sim_op_latent_append_t a) {
    const int half = a.rot_dim / 2;
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
    const int grid = (int)(a->tokens < (1 << 20) ? a->tokens : (1 << 20));
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) k_rotary<__nv_bfloat16><<<grid, 256, 0, st>>>(*a);
    else if (a->type == SIM_OP_FP16) k_rotary<__half><<<grid, 256, 0, st>>>(*a);
    else k_rotary<float><<<grid, 256, 0, st>>>(*a);
    return launched("sim_op_rotary");
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
    const int grid = (int)(a->tokens < (1 << 20) ? a->tokens : (1 << 20));
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->type == SIM_OP_BF16) k_append<__nv_bfloat16><<<grid, 128, 0, st>>>(*a);
    else if (a->type == SIM_OP_FP16) k_append<__half><<<grid, 128, 0, st>>>(*a);
    else k_append<float><<<grid, 128, 0, st>>>(*a);
    return launched("sim_op_latent_append");
}
