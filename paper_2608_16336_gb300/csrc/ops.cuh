// ops.cuh -- what the operators of an iteration share: argument errors,
// element types, rotary angles, warp sums.
#ifndef MTSIM_OPS_CUH
#define MTSIM_OPS_CUH

#include "mtsim_ops.h"

#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace mtop {

// Records the text for sim_op_last_error and gives the code back.
int fail(int code, const char *fmt, ...);

// The launch's error, or SIM_OK.
inline int launched(const char *what, cudaError_t e) {
    if (e == cudaSuccess) return SIM_OK;
    cudaGetLastError();  // the caller has it from here: it is not left for the next one that asks
    return fail(SIM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Lets a kernel use that much shared memory; `done` (one a kernel) keeps which devices have been told.
bool allow_shared(const void *kernel, int bytes, std::atomic<uint64_t> &done);

// Launches a kernel whose blocks may be set up while the one ahead of it in
// the stream still runs.  Every thread calls after_previous() before it reads
// or writes anything that is not its own, so that the stream's order holds;
// two calls in a row save 2 us of 15 to 100.
template <typename... P, typename... A>
inline cudaError_t launch_early(void (*kernel)(P...), unsigned grid, int threads, size_t shared, int cluster, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cfg.gridDim = dim3(grid), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = shared, cfg.stream = st;
    cfg.attrs = at, cfg.numAttrs = cluster > 1 ? 2 : 1;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// SMs of the current device (152 on a whole GB300), or 0 with an error set.
int sm_count();

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
// Whether the stride of a dimension is made of whole vectors of 16-bit elements; one of a single element says nothing.
inline bool even_stride(int64_t size, int64_t stride) { return size <= 1 || stride % 8 == 0; }

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

// 16 bytes of a row, and their elements in 32 bits.
template <typename T> struct alignas(16) Vec {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
    __device__ __forceinline__ void to(float *f) const {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = elem<T>::to(v[i]);
    }
    __device__ __forceinline__ void from(const float *f);
};
template <> __device__ __forceinline__ void Vec<float>::from(const float *f) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = f[i];
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16>::from(const float *f) {
#pragma unroll
    for (int i = 0; i < N; i += 2) *(__nv_bfloat162 *)(v + i) = __floats2bfloat162_rn(f[i], f[i + 1]);
}
template <> __device__ __forceinline__ void Vec<__half>::from(const float *f) {
#pragma unroll
    for (int i = 0; i < N; i += 2) *(__half2 *)(v + i) = __floats2half2_rn(f[i], f[i + 1]);
}

// Cosine and sine of position * frequency.  The angle in turns, modulo one,
// is position * (frequency / 2 pi * 2^64) in 64-bit wrapping integers: exact
// reduction at any position, one 64-bit multiplication an angle, and what is left is
// rounded once to 32 bits in [-1/2, 1/2) turns.  The factor is the frequency's
// 53-bit whole number times 2^66 / 2 pi, shifted by its exponent (64-bit
// floating point runs at a sixty-fourth of the rate here).
__device__ __forceinline__ unsigned long long turns_per_position(double frequency) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(frequency);
    const int e = (int)(b >> 52) & 0x7FF;
    const unsigned long long m = (b & 0xFFFFFFFFFFFFFull) | (e ? 1ull << 52 : 0);
    const unsigned long long c = 0xA2F9836E4E44152Aull;  // round(2^66 / 2 pi)
    const unsigned long long lo = m * c, hi = __umul64hi(m, c);
    const int right = 1077 - (e ? e : 1);  // (hi, lo) = turns * 2^64 * 2^right
    unsigned long long t;
    if (right <= 0) t = right > -64 ? lo << -right : 0;
    else if (right < 64) t = hi << (64 - right) | lo >> right;
    else t = right < 128 ? hi >> (right - 64) : 0;
    return b >> 63 ? 0 - t : t;
}

__device__ __forceinline__ void angle_cos_sin(unsigned long long turns, long long position, float &c, float &s) {
    const long long at = (long long)(turns * (unsigned long long)position);
    sincospif((float)(int)(at >> 32) * 4.656612873077393e-10f /* 2^-31: half turns */, &s, &c);
}

// The kernels before this one in the stream have ended and what they wrote is
// visible; the one after it may start (and wait here) from now on.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

}  // namespace mtop

#endif
