// block_copy.cu -- blocks of all layers to other blocks (mtsim_ops.h).
#include "ops.cuh"

namespace mtop {
namespace {

constexpr int kThreads = 256;

// V bytes at a time; a block of threads takes a pair in a layer.
template <typename V>
__global__ void __launch_bounds__(kThreads) k_block_copy(const __grid_constant__ sim_op_block_copy_t a) {
    let_next_start();
    after_previous();
    const int64_t units = (int64_t)a.pairs * a.layers, per_row = a.row_bytes / sizeof(V), all = per_row * a.rows;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t layer = u / a.pairs, i = u % a.pairs, from = a.from_blocks[i], to = a.to_blocks[i];
        if (from < 0 || from >= a.source_blocks || to < 0 || to >= a.destination_blocks) continue;
        const char *src = (const char *)a.source + layer * a.source_layer + from * a.source_block;
        char *dst = (char *)a.destination + layer * a.destination_layer + to * a.destination_block;
        for (int64_t k = threadIdx.x; k < all; k += kThreads) {
            const int64_t r = k / per_row, c = k % per_row * sizeof(V);
            *(V *)(dst + r * a.destination_row + c) = *(const V *)(src + r * a.source_row + c);
        }
    }
}

}  // namespace
}  // namespace mtop

using namespace mtop;

extern "C" int sim_op_block_copy(const sim_op_block_copy_t *given, void *stream) {
    if (!given) return fail(SIM_ERR_ARG, "args is NULL");
    sim_op_block_copy_t a = *given;
    if (a.layers < 0 || a.rows < 0 || a.pairs < 0 || a.row_bytes < 0 || a.source_blocks < 0 || a.destination_blocks < 0)
        return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a.layers == 0 || a.rows == 0 || a.pairs == 0 || a.row_bytes == 0 || a.source_blocks == 0 || a.destination_blocks == 0) return SIM_OK;
    if (!a.source || !a.destination || !a.from_blocks || !a.to_blocks)
        return fail(SIM_ERR_ARG, "source, destination, from_blocks and to_blocks must not be NULL");
    if (a.rows > 1 && (a.destination_row < a.row_bytes)) return fail(SIM_ERR_ARG, "destination rows must not overlap");
    // the stride of a dimension of one element is not used
    if (a.layers == 1) a.source_layer = a.destination_layer = 0;
    if (a.rows == 1) a.source_row = a.destination_row = 0;
    if (a.source_blocks == 1) a.source_block = 0;
    if (a.destination_blocks == 1) a.destination_block = 0;
    if (a.rows > 1 && a.source_row == a.row_bytes && a.destination_row == a.row_bytes) a.row_bytes *= a.rows, a.rows = 1;
    const int64_t bits = (int64_t)(uintptr_t)a.source | (int64_t)(uintptr_t)a.destination | a.row_bytes | a.source_layer | a.source_block | a.source_row |
                         a.destination_layer | a.destination_block | a.destination_row;
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    const int64_t units = (int64_t)a.pairs * a.layers, most = 8 * (int64_t)sms;
    const unsigned grid = (unsigned)(units < most ? units : most);
    cudaError_t e;
    if (bits % 16 == 0) e = launch_early(k_block_copy<uint4>, grid, kThreads, 0, 1, st, a);
    else if (bits % 4 == 0) e = launch_early(k_block_copy<uint32_t>, grid, kThreads, 0, 1, st, a);
    else e = launch_early(k_block_copy<uint8_t>, grid, kThreads, 0, 1, st, a);
    return launched("sim_op_block_copy", e);
}
