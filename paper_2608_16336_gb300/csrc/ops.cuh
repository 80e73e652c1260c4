// ops.cuh -- what the operators of an iteration share: argument errors,
// element types, rotary angles, warp sums.
#ifndef MTSIM_OPS_CUH
#define MTSIM_OPS_CUH

#include "mtsim_ops.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace mtop {

// Records the text for sim_op_last_error and gives the code back.
int fail(int code, const char *fmt, ...);

// The launch's error, or SIM_OK.
inline int launched(const char *what) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SIM_OK : fail(SIM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// SMs of the current device (152 on a whole GB300), or 0 with an error set.
int sm_count();

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

template <typename T> struct elem;
template <> struct elem<float> {
    static __device__ float to(float v) { return v; }
    static __device__ float from(float v) { return v; }
};
template <> struct elem<__nv_bfloat16> {
    static __device__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __nv_bfloat16 from(float v) { return __float2bfloat16(v); }
};
template <> struct elem<__half> {
    static __device__ float to(__half v) { return __half2float(v); }
    static __device__ __half from(float v) { return __float2half(v); }
};

// Cosine and sine of position * frequency.  The angle in turns, modulo one,
// is position * (frequency / 2 pi * 2^64) in 64-bit wrapping integers: exact
// reduction at any position, one 64-bit multiplication an angle, and what is left is
// rounded once to 32 bits in [-1/2, 1/2) turns.
__device__ __forceinline__ unsigned long long turns_per_position(double frequency) {
    const double t = frequency * 0.15915494309189533577;  // 1 / (2 pi)
    return __double2ull_rn((t - floor(t)) * 18446744073709551616.0);
}

__device__ __forceinline__ void angle_cos_sin(unsigned long long turns, long long position, float &c, float &s) {
    const long long at = (long long)(turns * (unsigned long long)position);
    sincospif((float)(int)(at >> 32) * 4.656612873077393e-10f /* 2^-31: half turns */, &s, &c);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

}  // namespace mtop

#endif
