// block_copy.cu -- blocks of all layers to other blocks (mtsim_ops.h).
#include "ops.cuh"

namespace mtop {
namespace {

// A block of threads takes a piece of a cache block at a time, V bytes a thread and kAhead of them on
// their way.  Rows that follow each other without a gap are one line.  Bound by memory: 640 blocks of 18 KB in 24 layers (566 MB
// read and written) take 84.1 us, 6.7 TB/s; 1,400 of 6.7 KB in 27 layers (508 MB) 76.2.
constexpr int kThreads = 128, kAhead = 4;

struct Pieces {
    uint32_t per_row, all, pieces;  // vectors of a row and of a block, pieces of a block
};

template <typename V, bool LINE>
__global__ void __launch_bounds__(kThreads) k_block_copy(const __grid_constant__ sim_op_block_copy_t a, const __grid_constant__ Pieces n) {
    let_next_start();
    after_previous();
    const uint64_t units = (uint64_t)a.pairs * a.layers * n.pieces;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint64_t block = n.pieces == 1 ? u : u / n.pieces;
        const uint32_t layer = (uint32_t)(block / (uint32_t)a.pairs), i = (uint32_t)(block - (uint64_t)layer * a.pairs);
        const int64_t from = a.from_blocks[i], to = a.to_blocks[i];
        if (from < 0 || from >= a.source_blocks || to < 0 || to >= a.destination_blocks) continue;
        const char *src = (const char *)a.source + layer * a.source_layer + from * a.source_block;
        char *dst = (char *)a.destination + layer * a.destination_layer + to * a.destination_block;
        const uint32_t k0 = (uint32_t)(u - block * n.pieces) * (kThreads * kAhead) + threadIdx.x;
        V v[kAhead];
        uint32_t row[kAhead], col[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const uint32_t k = k0 + e * kThreads;
            row[e] = LINE ? 0 : k / n.per_row, col[e] = (LINE ? k : k - row[e] * n.per_row);
            if (k < n.all) v[e] = *(const V *)(src + (LINE ? 0 : row[e] * a.source_row) + (size_t)col[e] * sizeof(V));
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (k0 + e * kThreads < n.all) *(V *)(dst + (LINE ? 0 : row[e] * a.destination_row) + (size_t)col[e] * sizeof(V)) = v[e];
    }
}

template <typename V> cudaError_t run(const sim_op_block_copy_t &a, cudaStream_t st) {
    const uint32_t per_row = (uint32_t)(a.row_bytes / sizeof(V)), all = per_row * (uint32_t)a.rows, step = kThreads * kAhead;
    const Pieces n = {per_row, all, (all + step - 1) / step};
    // a block of threads for every piece: with eight on each multiprocessor that go on, 94.8 and 93.8 us
    const uint64_t units = (uint64_t)a.pairs * a.layers * n.pieces, most = 1u << 30;
    const unsigned grid = (unsigned)(units < most ? units : most);
    return launch_early(a.rows == 1 ? k_block_copy<V, true> : k_block_copy<V, false>, grid, kThreads, 0, 1, st, a, n);
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
    if (a.rows > 1 && a.destination_row < a.row_bytes) return fail(SIM_ERR_ARG, "destination rows must not overlap");
    if (a.row_bytes > INT32_MAX || a.row_bytes * a.rows > INT32_MAX) return fail(SIM_ERR_ARG, "a block must have fewer than 2^31 bytes");
    // the stride of a dimension of one element is not used
    if (a.layers == 1) a.source_layer = a.destination_layer = 0;
    if (a.rows == 1) a.source_row = a.destination_row = 0;
    if (a.source_blocks == 1) a.source_block = 0;
    if (a.destination_blocks == 1) a.destination_block = 0;
    if (a.rows > 1 && a.source_row == a.row_bytes && a.destination_row == a.row_bytes) a.row_bytes *= a.rows, a.rows = 1, a.source_row = a.destination_row = 0;
    const int64_t bits = (int64_t)(uintptr_t)a.source | (int64_t)(uintptr_t)a.destination | a.row_bytes | a.source_layer | a.source_block | a.source_row |
                         a.destination_layer | a.destination_block | a.destination_row;
    const cudaStream_t st = (cudaStream_t)stream;
    return launched("sim_op_block_copy", bits % 16 == 0 ? run<uint4>(a, st)
                                         : bits % 8 == 0 ? run<uint2>(a, st)
                                         : bits % 4 == 0 ? run<uint32_t>(a, st)
                                                         : run<uint8_t>(a, st));
}
