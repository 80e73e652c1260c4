// tensor.cuh -- the fifth-generation tensor core, its memory, barriers and
// bulk copies, as inline PTX for sm_103a.
#ifndef MTSIM_TENSOR_CUH
#define MTSIM_TENSOR_CUH

#include "ops.cuh"

#include <cuda.h>

namespace mtop {

// ------------------------------------------------------------ barriers ----
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_retire(uint32_t bar) { asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// Waits that ran out, counted per source file (sim_op_faults adds them up): a kernel
// whose barrier never completes stops waiting after kWaitLimit tries
// (or kPollLimit polls: seconds), counts here and ends.
static __device__ unsigned g_faults;
constexpr int kWaitLimit = 1 << 22, kPollLimit = 1 << 26;

__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// The same without waiting at all, for a thread that has other work.
__device__ __forceinline__ bool bar_poll(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// Waits for the phase of that parity to complete; after a wait has run out,
// `dead` is set and later waits of the thread return at once.
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, bool &dead) {
    if (bar_test(bar, parity) || dead) return;
    for (int i = 0; i < kWaitLimit; ++i)
        if (bar_test(bar, parity)) return;
    dead = true;
    atomicAdd(&g_faults, 1u);
}

// ---------------------------------------------------------- bulk copies ---
__device__ __forceinline__ void copy_box_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void copy_box_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void fetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// Four rows anywhere in a 2-d tensor, the map's box being one row high.
__device__ __forceinline__ void copy_rows_4(uint32_t dst, const CUtensorMap *map, int x, int y0, int y1, int y2, int y3, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], "
        "[%7];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y0), "r"(y1), "r"(y2), "r"(y3), "r"(bar)
        : "memory");
}
// 16 bytes, or zeros where `real` is false.
__device__ __forceinline__ void copy_16(uint32_t dst, const void *src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_16_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Generic writes to shared memory become visible to the tensor core and to bulk copies.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// -------------------------------------------------------- tensor memory ---
__device__ __forceinline__ void tmem_alloc(uint32_t where, int cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, int cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: register c of lane l is column at + c of the warp's lane l.
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
        "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]),
        "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at)
        : "memory");
}

// COLS columns of 16 lanes (the first or second half of the warp's 32), in the
// register layout of a matrix fragment: registers 4k and 4k+1 of lane l are
// columns 8k + 2 (l % 4) and the next of row l / 4, registers 4k+2 and 4k+3 of row l / 4 + 8.
template <int COLS> __device__ __forceinline__ void tmem_ld_rows(uint32_t at, uint32_t *r);
template <> __device__ __forceinline__ void tmem_ld_rows<32>(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at)
                 : "memory");
}
template <> __device__ __forceinline__ void tmem_ld_rows<64>(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_st_rows64(uint32_t at, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x8.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at)
                 : "memory");
}

// ---------------------------------------------------------- tensor core ---
// A shared-memory operand in 128-byte-swizzled rows: 8 rows of 128 bytes make
// a 1,024-byte atom.  With K along the rows (64 16-bit elements a row),
// `stride` is the distance of 8-row groups along M or N, and a step of 16 along
// K adds 32 bytes to the address.  With M or N along the rows, `stride`
// is the distance of 8-row groups along K, and `lead` that of 64-element groups along M or N.
//
// The low word holds the address (which steps, in units of 16 bytes) and
// `lead`, the high word the rest, so that a step is one 32-bit addition.
__device__ __forceinline__ uint32_t operand_low(uint32_t addr, uint32_t lead) { return (addr >> 4 & 0x3FFF) | lead >> 4 << 16; }
__host__ __device__ constexpr uint32_t operand_high(uint32_t stride) { return stride >> 4 | 1u << 14 | 2u << 29; }

// One thread of a converged warp.  The tensor core takes its operands from
// registers that a warp has in common, and under this instruction's
// predicate (unlike `lane == 0`) the compiler keeps them there.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0;
}

// Instruction word of a product of 16-bit types into 32-bit sums.
__host__ __device__ constexpr uint32_t product_word(int m, int n, bool bf16, bool b_rows_along_n, bool negate_a) {
    return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (negate_a ? 1u << 13 : 0u) | (b_rows_along_n ? 1u << 16 : 0u) |
           (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

template <uint32_t A_HIGH, uint32_t B_HIGH>
__device__ __forceinline__ void product_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t word, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %6};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(word), "r"((uint32_t)add), "n"(A_HIGH),
        "n"(B_HIGH)
        : "memory");
}
// A in tensor memory (two 16-bit elements a column).
template <uint32_t B_HIGH>
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t word, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n mov.b64 b, {%2, %5};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(word), "r"((uint32_t)add), "n"(B_HIGH)
        : "memory");
}
// The barrier gets one arrival when every product this thread has queued is done.
__device__ __forceinline__ void product_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Registers of every thread of the warpgroup, within what the block was launched with.
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Every thread of every block of the cluster.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ------------------------------------------------------------ arithmetic --
// 2^x to about 2^-22 of itself, results below 2^-126 as 0: finer than the
// weights are rounded (2^-9, 2^-12), and one instruction where the full function is several.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two 32-bit operations in one instruction.
__device__ __forceinline__ void fma2(float &x0, float &x1, float a0, float a1, float b0, float b1, float c0, float c1) {
    asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
        " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}"
        : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void add2(float &x0, float &x1, float a0, float a1) {
    asm("{\n .reg .b64 a, d;\n mov.b64 a, {%2, %3};\n mov.b64 d, {%0, %1};\n add.rn.f32x2 d, d, a;\n mov.b64 {%0, %1}, d;\n}"
        : "+f"(x0), "+f"(x1) : "f"(a0), "f"(a1));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Pairs of 16-bit numbers.  spoil() adds 0 times a pair: 0 stays 0 unless a
// number is infinite or NaN.  finite_only() puts zeros in the place of such.
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    typedef __nv_bfloat162 two;
    static constexpr uint32_t exponent = 0x7F80;
};
template <> struct Pair<__half> {
    typedef __half2 two;
    static constexpr uint32_t exponent = 0x7C00;
};
template <typename T> __device__ __forceinline__ void spoil(uint32_t &sum, uint32_t w) {
    typedef typename Pair<T>::two two;
    const uint32_t zero = 0;
    *(two *)&sum = __hfma2(*(const two *)&w, *(const two *)&zero, *(two *)&sum);
}
__device__ __forceinline__ bool spoiled(uint32_t sum) { return sum & 0x7FFF7FFF; }
template <typename T> __device__ __forceinline__ uint32_t finite_only(uint32_t w) {
    constexpr uint32_t e = Pair<T>::exponent;
    return w & ((w & e) == e ? 0xFFFF0000u : ~0u) & ((w >> 16 & e) == e ? 0xFFFFu : ~0u);
}

// How softmax weights are held as an operand of the product with the values.
// They are exp2(s - m + raise) for a maximum m that is taken anew when it has
// grown by 2^grow, so the largest is below 2^(raise + grow).  bfloat16 has the
// range of 32 bits.  float16 ends at 2^-24 (2^-14 with all of its bits), so there
// the weights use the range above 1 too: one is rounded by at most 2^-35 of
// the largest, where without the raise all below 2^-25 of it were lost (0.4 % of a row's weight
// in 130,000 tokens).  raise + grow leave a factor 2 to the type's end.
// 3 requests of 90,001 to 130,000 tokens take 89 us with 5, 92 with 4 (88 without the raise and 8).
template <typename T> struct WeightRange {
    static constexpr float raise = 0.f, grow = 8.f;
};
template <> struct WeightRange<__half> {
    static constexpr float raise = 10.f, grow = 5.f;
};

// s - m is a product and a sum rounded once, so it may lie above 0 by what m,
// the scaled maximum, was rounded by: below one half up to this size (beyond it
// the weights would leave the type).  Larger ones are rounded as m was before m is taken off.
constexpr float kFusedUpTo = 8388608.f;
__device__ __forceinline__ bool beyond_fused(float top) { return fabsf(top) > kFusedUpTo; }  // or -infinity: nothing seen
__device__ __forceinline__ float below_top(float x, float scale, float top) {
    return __fsub_rn(__fmul_rn(x, scale), top == -INFINITY ? 0.f : top);
}

// A tensor map of `dims` dimensions (the first contiguous) of 16-bit
// elements in 128-byte-swizzled boxes; false with the error set when the
// driver refuses it.  strides: elements, of dimensions 1 and up.
bool box_map(CUtensorMap *map, const void *base, bool bf16, int dims, const uint64_t *size, const int64_t *stride, const uint32_t *box);

}  // namespace mtop

#endif
