// ops.cu -- what the operators' host sides share (ops.cuh).
#include "tensor.cuh"

#include <atomic>
#include <cstdarg>
#include <cstdio>

#include <cudaTypedefs.h>

namespace mtop {

namespace {
thread_local char t_error[512] = "";
}

int fail(int code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(t_error, sizeof t_error, fmt, ap);
    va_end(ap);
    return code;
}

int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev < 64 && known[dev].load(std::memory_order_relaxed)) return known[dev].load(std::memory_order_relaxed);
    int n = 0;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) {
        fail(SIM_ERR_CUDA, "device query: %s", cudaGetErrorString(e));
        return 0;
    }
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

bool allow_shared(const void *kernel, int bytes, std::atomic<uint64_t> &done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (e == cudaSuccess && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) {
        fail(SIM_ERR_CUDA, "shared memory: %s", cudaGetErrorString(e));
        return false;
    }
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

namespace {
bool make_map(CUtensorMap *map, const void *base, CUtensorMapDataType type, int bytes, int dims, const uint64_t *size, const int64_t *stride,
              const uint32_t *box) {
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> encode{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 f = encode.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        void *p = nullptr;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess || found != cudaDriverEntryPointSuccess || !p) {
            fail(SIM_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
            return false;
        }
        f = (PFN_cuTensorMapEncodeTiled_v12000)p;
        encode.store(f, std::memory_order_release);
    }
    cuuint64_t strides[4];
    cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    for (int d = 0; d + 1 < dims; ++d) strides[d] = (cuuint64_t)stride[d] * bytes;
    const CUresult r = f(map, type, (cuuint32_t)dims, const_cast<void *>(base), (const cuuint64_t *)size, strides, box, ones,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, box[0] * bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) fail(SIM_ERR_CUDA, "tensor map: driver error %d", (int)r);
    return r == CUDA_SUCCESS;
}
}  // namespace

bool box_map(CUtensorMap *map, const void *base, bool bf16, int dims, const uint64_t *size, const int64_t *stride, const uint32_t *box) {
    return make_map(map, base, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, dims, size, stride, box);
}
bool byte_box_map(CUtensorMap *map, const void *base, int dims, const uint64_t *size, const int64_t *stride, const uint32_t *box) {
    return make_map(map, base, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, dims, size, stride, box);
}

unsigned decode_faults();
unsigned prefill_faults();
unsigned quantized_faults();

}  // namespace mtop

extern "C" int sim_op_faults(void) {
    // (a copy alone would not wait for streams that do not wait for the default one)
    const cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return mtop::launched("sim_op_faults", e);
    const unsigned d = mtop::decode_faults(), p = mtop::prefill_faults(), q = mtop::quantized_faults(), n = d + p + q;
    return d == ~0u || p == ~0u || q == ~0u || n > 0x7FFFFFFFu ? mtop::fail(SIM_ERR_CUDA, "the fault counter cannot be read") : (int)n;
}

extern "C" const char *sim_op_last_error(void) { return mtop::t_error; }
