// quantized_decode.cu -- attention of new tokens over the 8-bit block cache
// of latent vectors (mtsim_ops.h).
#include "eight.cuh"
#include "tensor.cuh"

#include <cmath>

namespace mtop {
namespace {

// The cached bytes are operands as they are: the tensor core multiplies 8-bit
// floats, and nothing is unpacked.  A block takes R = 16 or 32 rows (new token x head) of a request,
// over tiles of 64 cached tokens, with tokens (then latent elements) along the product's rows:
//   S^T = C Q^T            (64 tokens x R, latent and key part apart)
//   P = exp2(S - m)
//   O^T += C[:, :rank]^T P (rank x R, in products of 128 elements)
// A tile is one operand twice: tokens along the rows for S^T, and the same bytes read across them for O^T.
//
// Queries and weights have more bits than 8-bit floats, so each is a sum of such
// floats, side by side along the product's columns (a wider product costs little: it is bound by
// reading C from shared memory).  A query row, times a power of two that brings its largest to
// [128, 256), is e4m3 + e4m3 / 16 (+ e4m3 / 256): exact for 16-bit types down to 2^-14 of the largest.
// A weight, at most 2^15, is e5m2 + e5m2 / 8 + e5m2 / 64 (+ e5m2 / 512).  e5m2 is the upper half of a 16-bit float, so the
// terms are cut from one with whole-number operations.
//
// The weight that multiplies c is exp2(s) a, for the latent scale a of the token's block; its exponent is s + log2 a, so
// that the running maximum is that of the products and they keep the type's range, and the
// softmax's sum takes each divided by a again.
//
// Bound by shared memory, of whose 128 bytes a cycle a tile of 32 rows and 576 bytes a token takes 1,390 cycles' worth (the copy 290, C 580, once
// for the scores and once for the sums, Q 290, P 190 and its way there), by the way from scores to weights, which a tile's warps go one tile after another, and by
// the steps of the one thread that queues the products (1,800 to 2,000 cycles a tile in all).  64 requests of 200 to 10,240 tokens, 128 heads (122 MB, 50 GFLOP): 114.5 us, 134 before requests'
// costs were counted in the parts.  3 requests of 90,001 to 130,000 tokens, two new ones, 16 heads (204 MB): 81.
// Tiles of 128 tokens read Q half as often and have half the steps, but two stages are too few: 161 and 118 us.
constexpr int kTile = 64, kUnit = 32;   // tokens of a tile, and of what a part may begin and end with
constexpr int kColBytes = kTile * 128;  // a stage's column block: 64 tokens x 128 bytes
constexpr int kSide = 16;               // rows side by side in a term of P
constexpr int kGroup = 8;               // rows of a warpgroup (16: a longer chain from scores to weights, 82.7 us for the long requests, 14.0 instead of 13.0 for one of 777 tokens)
constexpr int kWeights = 3;             // buffers of P
constexpr int kMostStages = 8;
constexpr int kShared = 227 * 1024;
constexpr int kCols = 512;
// A warp hands over its copies one after another (70 cycles each): 128 tokens in boxes of 16
// come in 1.1 us from three warps, in 2.0 from one.
constexpr int kCopyWarps = 3, kScaleWarps = kTile / 32;
constexpr int kPieces = 16;  // row factors are kept of so many pieces: queries are made ready while as many as all stages and three more are under way
constexpr float kRaise = 5.f, kLimit = 15.f;  // weights are exp2(y - max + raise), the maximum taken anew beyond the limit
constexpr float kNothing = 3e38f;              // raise - max of a row that has seen nothing

// Terms of queries and weights.
template <typename T> struct Terms {
    static constexpr int q = 2, p = 3;
};
template <> struct Terms<__half> {
    static constexpr int q = 3, p = 4;
};
template <typename T, int G> struct Shape {
    static constexpr int rows = G * kGroup, nq = Terms<T>::q * rows, np = Terms<T>::p * rows;
    static constexpr int soft = 4 * G, threads = (soft + 1 + kCopyWarps + 4) * 32;  // + products, copies, queries
    static constexpr int chunk = nq * 16 + 16;  // bytes of Q from 16 elements to the next (a bank's width apart)
    static constexpr int p_bytes = np * kTile;  // [np / 16][64 tokens][16]
    static constexpr int s_at = 4 * np;         // columns; S^T's two buffers are the halves of the lanes
    static_assert(s_at + 2 * nq <= kCols, "tensor memory");
};
constexpr uint32_t kUpper = 16u << 16;  // the second 16 lanes of each 32

struct Args {
    const void *q;
    const float *scales;
    const int32_t *table, *lengths;
    void *out;
    float *lse;
    int *first;     // [requests + 1]: where each request begins on the line
    float *sums;    // [parts][2][R][rank]: the unfinished O of a part's first and last piece
    float2 *stats;  // [parts][2][R]: raise - maximum, and sum of weights
    int64_t q_request, q_token, q_head, out_request, out_token, out_head, table_row;
    int64_t blocks, most;  // most: tokens a table can name
    int requests, new_tokens, heads, rank, width;
    int block_tokens, row_ratio;  // cache_block / cache_row
    int row_tiles, lanes;         // parts = row_tiles * lanes
    int stages;
    int run;         // tokens a copy takes
    bool scattered;  // four rows anywhere instead of a run
    bool thin;       // the key part alone is the last column block: 64 bytes of it are kept
    int none;        // a row outside the cache
    float scale_log2;
};

template <int R> struct Barriers {
    uint64_t full[kMostStages], empty[kMostStages], q_full, q_empty, s_ready[2], p_ready[2], pv_done[4], o_free;
    uint32_t tmem;
    int first_request, first_unit, total, late;
    float2 scale[kMostStages][kTile];
    alignas(16) float factor[kPieces][R];
    alignas(16) float met[R / kGroup][4][kGroup], keep[R / kGroup][kGroup];
    int64_t to[R];
    int later[R];  // new tokens after the row's own one
};
__device__ __forceinline__ int tokens_of(const Args &a, int b) { return (int)min(max((int64_t)a.lengths[b], (int64_t)0), a.most); }
// A request's stretch on the line of all requests, which is cut into the blocks' parts: its units, after
// as many as a request costs a part besides (its queries, the first tile's start, its sums' way out).  Of the times of a call's
// parts: 6 to 6.5 us with 32 rows, where a tile of two units takes 1.07; with 16 rows 3 and 0.85, or 7 units, too few to matter.
constexpr int kRequestUnits = 12;
__device__ __forceinline__ int line_of(int tokens) { return tokens ? (tokens + kUnit - 1) / kUnit + kRequestUnits : 0; }

// Parts in use and where one begins on the line.
__device__ __forceinline__ int parts_of(const Args &a, int total) {
    return max(1, min(a.lanes, min(total, (int)(5.f * __fsqrt_rn((float)total * a.requests)))));
}
__device__ __forceinline__ int begin_of(int total, int parts, int p) {  // floor(total * p / parts)
    return p < parts ? total / parts * p + total % parts * p / parts : total;
}

// The tiles of a part, piece by piece: request b, units [u0, u1) of its n, the tile that begins at unit u.
struct Walk {
    int b, u0, u1, n, u, left, piece, tokens;
    int at;     // where the piece begins in the request's stretch
    int after;  // the next request's tokens, read ahead
    bool more;
    __device__ void start(const Args &a, int b0, int offset, int count) {
        b = b0, at = offset, left = count, piece = 0, after = tokens_of(a, b0);
        more = settle(a);
    }
    __device__ bool settle(const Args &a) {
        if (left <= 0) return false;
        while (true) {
            tokens = after, n = (tokens + kUnit - 1) / kUnit;
            if (b + 1 < a.requests) after = tokens_of(a, b + 1);
            else if (n == 0) return false;
            if (n) break;
            ++b;  // the part goes on, so a request with some follows
        }
        u0 = max(at - kRequestUnits, 0), u1 = min(n, at + left - kRequestUnits), u = u0;
        return u1 > u0;  // (else the part ends before the request's first)
    }
    __device__ int tiles() const { return more ? (u1 - u0 + kTile / kUnit - 1) / (kTile / kUnit) : 0; }
    __device__ int past() const { return min(tokens, kUnit * u1); }
    __device__ bool last() const { return u + kTile / kUnit >= u1; }
    __device__ void next_piece(const Args &a) {
        left -= u1 + kRequestUnits - at, ++b, at = 0, ++piece;
        more = b < a.requests && settle(a);
    }
    __device__ void next(const Args &a) {
        if (last()) next_piece(a);
        else u += kTile / kUnit;
    }
};

// 8 columns of the warp's 32 lanes.
__device__ __forceinline__ void tmem_ld8(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(at)
                 : "memory");
}
// 8 columns of 16 lanes: a lane has columns 2q and 2q + 1, q = lane % 4, of lane / 4 and of 8 further.
__device__ __forceinline__ void tmem_ld_rows8(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// Products of 8-bit floats into 32-bit sums.  C is in 128-byte-swizzled rows, a token
// each: with tokens along the product's rows, 8 of them are 1,024 bytes, and a step of 32 elements adds 32
// bytes; read across, the row of 128 elements is a product's, 8 tokens are 1,024 bytes, and a step of 32 tokens adds 4,096.
// Q and P are not swizzled, but made of 8 x 16 bytes: Q's 16 elements of 8 rows, P's 16 rows of 8 tokens.
constexpr uint32_t kHighC = operand_high(1024), kHighKey = 512u >> 4 | 1u << 14 | 4u << 29;  // (a thin key part: rows of 64 bytes, swizzled within these)
__host__ __device__ constexpr uint32_t plain_high(uint32_t stride) { return stride >> 4 | 1u << 14; }
__host__ __device__ constexpr uint32_t word_8(int m, int n, bool a_across, bool b_e5m2, bool b_across) {
    return 1u << 4 | (b_e5m2 ? 1u << 10 : 0u) | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
template <uint32_t A_HIGH, uint32_t B_HIGH>
__device__ __forceinline__ void product_8(uint32_t d, uint32_t a, uint32_t b, uint32_t word, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %6};\n"
        " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(word), "r"((uint32_t)add), "n"(A_HIGH),
        "n"(B_HIGH)
        : "memory");
}
// N products in a row, of operands that lie STEP_A and STEP_B bytes apart.  (The thread that issues them
// has few instructions for each: with the addresses worked out one by one S^T took 900 cycles to issue and 540 to compute.)
template <int N, uint32_t A_HIGH, uint32_t B_HIGH, int STEP_A, int STEP_B>
__device__ __forceinline__ void products_8(uint32_t d, uint32_t a, uint32_t b, uint32_t word, bool add) {
    product_8<A_HIGH, B_HIGH>(d, a, b, word, add);
#pragma unroll
    for (int k = 1; k < N; ++k) product_8<A_HIGH, B_HIGH>(d, a + (STEP_A >> 4) * k, b + (STEP_B >> 4) * k, word, true);
}

// Every thread of the group, and whether one of them says yes.
__device__ __forceinline__ void group_sync(int g) { asm volatile("bar.sync %0, 128;" ::"r"(g + 1) : "memory"); }
__device__ __forceinline__ bool group_any(int g, bool yes) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}"
                 : "=r"(r) : "r"((uint32_t)yes), "r"(g + 1) : "memory");
    return r != 0;
}

// The larger magnitude of two 16-bit numbers, as a 32-bit one's bits.
template <typename T> __device__ __forceinline__ uint32_t size_bits(uint32_t two) {
    const uint32_t size = two & 0x7FFF7FFF;
    const uint32_t more = max(size & 0xFFFF, size >> 16);
    const T v = *(const T *)&more;
    return __float_as_uint(elem<T>::to(v)) & 0x7FFFFFFF;
}

// A lane's two rows, joined over the lanes that have them too.
template <typename F> __device__ __forceinline__ void join2(float *v, F f) {
#pragma unroll
    for (int bit = 4; bit < 32; bit *= 2)
#pragma unroll
        for (int e = 0; e < 2; ++e) v[e] = f(v[e], __shfl_xor_sync(~0u, v[e], bit));
}

// A byte that is NaN becomes zero: the weight of a row that does not see it is 0, and 0 times NaN is not.
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
    const uint32_t nan = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    return w & ~((nan >> 7) * 0xFFu);
}

template <typename T, int G>
__global__ void __launch_bounds__(Shape<T, G>::threads, 1) k_quantized_decode(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap m_cache, const __grid_constant__ CUtensorMap m_key) {
    using Z = Shape<T, G>;
    constexpr int R = Z::rows, QT = Terms<T>::q, PT = Terms<T>::p;
    using Bars = Barriers<R>;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int cols = (a.width + 127) / 128, steps = (a.width + 31) / 32, latent_steps = a.rank / 32, stage_bytes = cols * kColBytes - (a.thin ? kColBytes / 2 : 0);
    const int tiles_m = (a.rank + 127) / 128;
    const int q_offset = a.stages * stage_bytes, p_offset = q_offset + 2 * steps * Z::chunk;
    const uint32_t stage_at = smem_addr(smem), q_at = stage_at + q_offset, p_at = stage_at + p_offset;
    Bars *bars = (Bars *)(smem + p_offset + kWeights * Z::p_bytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rt = blockIdx.x % a.row_tiles, part = blockIdx.x / a.row_tiles;
    const int rows = a.new_tokens * a.heads, here = min(R, rows - rt * R);
    bool dead = false;
    let_next_start();

    if (warp == 1 && lane == 0) {
#pragma unroll 1
        for (int s = 0; s < a.stages; ++s) bar_init(smem_addr(&bars->full[s]), kCopyWarps + kScaleWarps), bar_init(smem_addr(&bars->empty[s]), 1);
        bar_init(smem_addr(&bars->q_full), 128);
        bar_init(smem_addr(&bars->q_empty), 1);
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&bars->s_ready[s]), 1);
            bar_init(smem_addr(&bars->p_ready[s]), 128 * G);
        }
        for (int s = 0; s < 4; ++s) bar_init(smem_addr(&bars->pv_done[s]), 1);
        bar_init(smem_addr(&bars->o_free), 128 * G);
        bars->late = 0;
        bar_init_done();
    }
    if (warp == Z::soft) tmem_alloc(smem_addr(&bars->tmem), kCols);
    if (warp > Z::soft && warp < Z::soft + 1 + kCopyWarps && lane == 0) fetch_map(&m_cache), fetch_map(&m_key);
    if (warp >= Z::soft + 1 + kCopyWarps) {
        const int r = threadIdx.x - (Z::soft + 1 + kCopyWarps) * 32;
        if (r < R) {
            const int flat = min(rt * R + r, rows - 1), tok = flat / a.heads;
            bars->to[r] = tok * a.out_token + (flat - tok * a.heads) * a.out_head;
            bars->later[r] = a.new_tokens - 1 - tok;
        }
    }
    __syncwarp();
    after_previous();
    if (warp == 0) {
        // the line's length, and where this part begins on it
        int total = 0, kept[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) kept[k] = 32 * k + lane < a.requests ? line_of(tokens_of(a, 32 * k + lane)) : 0, total += kept[k];
#pragma unroll 1
        for (int b0 = 128; b0 < a.requests; b0 += 32) total += b0 + lane < a.requests ? line_of(tokens_of(a, b0 + lane)) : 0;
        total = (int)__reduce_add_sync(~0u, (unsigned)total);
        const int begin = begin_of(total, parts_of(a, total), part);
        int seen = 0;
        auto place = [&](int b0, int n) {
            int incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl += u;
            }
            const int at = seen + incl - n;
            if (n && begin >= at && begin < at + n) bars->first_request = b0 + lane, bars->first_unit = begin - at;
            if (blockIdx.x == 0 && b0 + lane < a.requests) a.first[b0 + lane] = at;
            seen += __shfl_sync(~0u, incl, 31);
        };
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (32 * k < a.requests) place(32 * k, kept[k]);
#pragma unroll 1
        for (int b0 = 128; b0 < a.requests; b0 += 32) place(b0, b0 + lane < a.requests ? line_of(tokens_of(a, b0 + lane)) : 0);
        if (lane == 0) {
            bars->total = total;
            if (blockIdx.x == 0) a.first[a.requests] = total;
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = bars->tmem;
    const int parts = parts_of(a, bars->total);
    const int begin = begin_of(bars->total, parts, part), end = begin_of(bars->total, parts, part + 1);
    Walk w;
    w.start(a, end > begin ? bars->first_request : 0, end > begin ? bars->first_unit : 0, end - begin);

    if (warp >= Z::soft + 1 + kCopyWarps) {
        // ------------------------------------------------ queries and scales
        // a warp takes four rows at a time, its lanes 8 elements of each; then the first
        // two a tile's scales, a token a thread, with the next tile's on their way
        const int vectors = 4 * steps, w0 = warp - (Z::soft + 1 + kCopyWarps), token = threadIdx.x - (Z::soft + 1 + kCopyWarps) * 32;
        int s = 0;
        uint32_t round = 0;
        for (int k = 0; w.more; w.next_piece(a), ++k) {
            const T *q = (const T *)a.q + w.b * a.q_request;
            const int32_t *table = a.table + w.b * a.table_row;
            const int past = w.past();
            auto block_of = [&](int u) {
                const int j = kUnit * u + token;
                return token < kTile && j < past ? table[j / a.block_tokens] : -1;
            };
            auto scales_of = [&](int id) { return id >= 0 && id < a.blocks ? ((const float2 *)a.scales)[id] : make_float2(1.f, 1.f); };
            int id = block_of(w.u0);
            float2 ahead;
            auto row_at = [&](int r, uint4 *x) {
                const int flat = rt * R + r, tok = flat / a.heads;
                const T *from = q + tok * a.q_token + (flat - tok * a.heads) * a.q_head;
#pragma unroll
                for (int v = 0; v < 3; ++v) {
                    const int j = lane + 32 * v;
                    x[v] = r < R && flat < rows && 8 * j < a.width ? *(const uint4 *)(from + 8 * j) : make_uint4(0, 0, 0, 0);
                }
            };
            uint4 x[3], y[3];
            row_at(w0, x);
            ahead = scales_of(id), id = block_of(w.u0 + kTile / kUnit);
            bar_await(smem_addr(&bars->q_empty), (k & 1) ^ 1, dead);
            // (little code: it runs once a piece, and fetching it is most of what it costs)
#pragma unroll 1
            for (int r = w0; r < R; r += 4) {
                row_at(r + 4, y);
                uint32_t most = 0;
#pragma unroll
                for (int v = 0; v < 3; ++v) most = max(most, max(max(size_bits<T>(x[v].x), size_bits<T>(x[v].y)), max(size_bits<T>(x[v].z), size_bits<T>(x[v].w))));
                most = __reduce_max_sync(~0u, most);
                // the power of two that brings the largest to [128, 256) (as far as 32 bits hold it)
                const int up = most == 0 ? 0 : min(134 - (int)(most >> 23), 126);
                const float by = __uint_as_float((uint32_t)(up + 127) << 23), back = __uint_as_float((uint32_t)(127 - up) << 23);
                // infinities and NaN: the row is NaN
                if (lane == 0) bars->factor[k % kPieces][r] = most < 0x7F800000u ? a.scale_log2 * back : NAN;
                uint32_t to = q_at + lane / 2 * Z::chunk + (r / kSide * QT * kSide + r % kSide) * 16 + lane % 2 * 8;
#pragma unroll 1
                for (int j = lane; j < vectors; j += 32, to += 16 * Z::chunk) {
                    float f[8];
                    ((const Vec<T> *)x)->to(f);
                    // (up to 11 bits below 256 are a 16-bit float, and so is what a term leaves of them; one below 2^-14
                    // is rounded by at most 2^-25, far less than the last term can tell)
                    __half2 h[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = __floats2half2_rn(f[2 * e] * by, f[2 * e + 1] * by);
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        uint32_t two[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            two[e] = pack_e4m3(h[e]);
                            h[e] = __hmul2(__hsub2(h[e], halves_of_e4m3(two[e])), __floats2half2_rn(16.f, 16.f));
                        }
                        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to + t * kSide * 16), "r"(two[0] | two[1] << 16), "r"(two[2] | two[3] << 16) : "memory");
                    }
                    x[0] = x[1], x[1] = x[2];
                }
#pragma unroll
                for (int v = 0; v < 3; ++v) x[v] = y[v];
            }
            fence_async();
            bar_arrive(smem_addr(&bars->q_full));
            for (int u = w.u0; w0 < kScaleWarps && u < w.u1; u += kTile / kUnit) {
                const float2 now = ahead;
                ahead = scales_of(id), id = block_of(u + 2 * (kTile / kUnit));
                bar_await(smem_addr(&bars->empty[s]), (round & 1) ^ 1, dead);
                bars->scale[s][token] = make_float2(scale_used(now.x), scale_used(now.y));
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&bars->full[s]));
                if (++s == a.stages) s = 0, ++round;
            }
        }
    } else if (warp >= Z::soft) {
        if (warp > Z::soft) {
            // ----------------------------------------------------- cache copies
            // a copy takes `run` tokens of a block by 128 bytes, or, where blocks are
            // not whole multiples of 4 tokens, any four rows; every third is this warp's
            const int run = a.run, groups = kTile / run, copies = groups * cols, mine = warp - Z::soft - 1;
            const int thin_at = a.thin ? copies - groups : copies;  // copies from there on take 64 bytes a row
            uint32_t bytes = 0;
#pragma unroll 1
            for (int n = mine; n < copies; n += kCopyWarps) bytes += run * (n < thin_at ? 128 : 64);
            int s = 0;
            uint32_t round = 0;
            for (; w.more; w.next(a)) {
                const int past = w.past();
                const int32_t *table = a.table + w.b * a.table_row;
                const uint32_t full = smem_addr(&bars->full[s]);
                bool waited = false;
#pragma unroll 1
                for (int n0 = mine; n0 < copies; n0 += 32 * kCopyWarps) {
                    const int n = n0 + kCopyWarps * lane, c = n / groups, group = n - c * groups;
                    int row[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = kUnit * w.u + run * group + e;
                        row[e] = a.none;
                        if ((e == 0 || a.scattered) && j < past && n < copies) {
                            const int blk = j / a.block_tokens, id = table[blk];
                            if (id >= 0 && id < a.blocks) row[e] = id * a.row_ratio + (j - blk * a.block_tokens);
                        }
                    }
                    if (!waited) {
                        bar_await(smem_addr(&bars->empty[s]), (round & 1) ^ 1, dead);
                        if (lane == 0) bar_expect(full, bytes);
                        __syncwarp();
                        waited = true;
                    }
                    const uint32_t dst = stage_at + s * stage_bytes + c * kColBytes + group * run * (n < thin_at ? 128 : 64);
                    const CUtensorMap *map = n < thin_at ? &m_cache : &m_key;
                    if (n < copies) {
                        if (a.scattered) copy_rows_4(dst, map, 128 * c, row[0], row[1], row[2], row[3], full);
                        else copy_box_2d(dst, map, 128 * c, row[0], full);
                    }
                }
                if (++s == a.stages) s = 0, ++round;
            }
        } else {
            // -------------------------------------------------------- products
            constexpr uint32_t word_s = word_8(kTile, Z::nq, false, false, false), word_p = word_8(128, Z::np, true, true, true);
            constexpr uint32_t high_q = plain_high(128), high_p = plain_high(kTile * 16);
            auto scores = [&](int i, int s) {
                const uint32_t d = tmem + Z::s_at + (i & 1 ? kUpper : 0);
                constexpr int step_q = 2 * Z::chunk;
                uint32_t q_low = operand_low(q_at, Z::chunk), c_low = operand_low(stage_at + s * stage_bytes, 16);
                bool add = false;
#pragma unroll 1
                for (int k = 4; k <= latent_steps; k += 4, c_low += kColBytes >> 4, q_low += 4 * step_q >> 4, add = true)
                    products_8<4, kHighC, high_q, 32, step_q>(d, c_low, q_low, word_s, add);
                if (latent_steps % 4) products_8<2, kHighC, high_q, 32, step_q>(d, c_low, q_low, word_s, add), c_low += 64 >> 4, q_low += 2 * step_q >> 4;
                const int key_steps = steps - latent_steps;
                if (a.thin) {
                    if (key_steps == 2) products_8<2, kHighKey, high_q, 32, step_q>(d + Z::nq, c_low, q_low, word_s, false);
                    else product_8<kHighKey, high_q>(d + Z::nq, c_low, q_low, word_s, false);
                } else if (key_steps == 2) products_8<2, kHighC, high_q, 32, step_q>(d + Z::nq, c_low, q_low, word_s, false);
                else if (key_steps == 1) product_8<kHighC, high_q>(d + Z::nq, c_low, q_low, word_s, false);
                product_commit(smem_addr(&bars->s_ready[i & 1]));
            };
            auto weighted = [&](int i, int buffer, int s, bool add) {
                const uint32_t p_low = operand_low(p_at + buffer * Z::p_bytes, 128);
                uint32_t c_low = operand_low(stage_at + s * stage_bytes, 16), d = tmem;
#pragma unroll 1
                for (int m = 0; m < tiles_m; ++m, c_low += kColBytes >> 4, d += Z::np)
                    products_8<kTile / 32, kHighC, high_p, 4096, 32 * 16>(d, c_low, p_low, word_p, add);
                product_commit(smem_addr(&bars->empty[s]));
                product_commit(smem_addr(&bars->pv_done[i & 3]));
            };
            // One thread does it all.  When a tile's weights are there, the scores of the next but one are queued (S^T's
            // buffer is free: the weights were made from it), then this tile's sums, so that the next
            // weights never wait for their scores.  A tile's scores come after the sums of three tiles before, so when
            // they are there, its buffer of P is free.  A look at a barrier and every step of this loop take 100 to 400 cycles (the
            // tensor core has the shared memory, the others' code the instruction caches), so there are few of them:
            // 64 requests, 128 heads take 114 us, with three barriers a tile and the sums first 148.
            Walk ws = w;
            int si = 0, s_left = ws.tiles(), w_left = s_left, s_stage = 0, w_stage = 0, buffer = 0;
            uint32_t s_round = 0;
            bool q_here = false, add = false;
            const bool elected = elect_one();
            auto queue_scores = [&]() {
                tmem_after_sync();
                scores(si, s_stage);
                ++si;
                if (++s_stage == a.stages) s_stage = 0, ++s_round;
                if (--s_left == 0) {
                    product_commit(smem_addr(&bars->q_empty));
                    ws.next_piece(a);
                    s_left = ws.tiles(), q_here = false;
                }
            };
            for (int wi = 0; elected && w_left; ++wi) {
                while (s_left && si < wi + 2) {
                    if (!q_here) {
                        // (of the next piece: not waited for while sums can be queued)
                        if (wi < si && !bar_poll(smem_addr(&bars->q_full), ws.piece & 1)) break;
                        bar_await(smem_addr(&bars->q_full), ws.piece & 1, dead);
                        q_here = true;
                    }
                    bar_await(smem_addr(&bars->full[s_stage]), s_round & 1, dead);
                    queue_scores();
                }
                bar_await(smem_addr(&bars->p_ready[wi & 1]), (wi / 2) & 1, dead);
                if (q_here && si == wi + 2 && bar_poll(smem_addr(&bars->full[s_stage]), s_round & 1)) queue_scores();
                if (!add && w.piece > 0) bar_await(smem_addr(&bars->o_free), (w.piece - 1) & 1, dead);
                tmem_after_sync();
                weighted(wi, buffer, w_stage, add);
                if (++w_stage == a.stages) w_stage = 0;
                if (++buffer == kWeights) buffer = 0;
                add = --w_left != 0;
                if (!add) w.next_piece(a), w_left = w.tiles();
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------- weights and sums
        // a lane has two tokens, 8 apart, and two rows
        const int g = warp / 4, q = lane % 4, t0 = warp % 4 * 16 + lane / 4;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t side = g % 2 * kGroup, s_at = tmem + Z::s_at + lanes + g / 2 * QT * kSide + side, o_at = tmem + lanes + g / 2 * PT * kSide + side;
        const bool with_key = a.width > a.rank;
        // a tile's sums (a barrier tells one phase from the one before only: those of four tiles before are known to be there, as
        // a tile's scores come after the sums of three before)
        auto pv_wait = [&](int j) { bar_await(smem_addr(&bars->pv_done[j & 3]), (j / 4) & 1, dead); };
        auto larger = [](float x, float z) { return fmaxf(x, z); };
        auto added = [](float x, float z) { return x + z; };
        int later[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) later[e] = bars->later[g * kGroup + 2 * q + e];
        float base[2], sum[2];
        int stage = 0, buffer = 0;
        uint32_t round = 0;
        for (int i = 0; w.more; ++i) {
            if (w.u == w.u0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) base[e] = kNothing, sum[e] = 0.f;
            }
            const int tokens = w.tokens, fewest = tokens - a.new_tokens + 1, j0 = kUnit * w.u, past = w.past();
            float y[2][2], per_sl[2];
            {
                bar_await(smem_addr(&bars->s_ready[i & 1]), (i / 2) & 1, dead);
                tmem_after_sync();
                // [term][token, 8 tokens on][two rows]
                uint32_t l[QT][4], c[QT][4];
                const uint32_t from = s_at + (i & 1 ? kUpper : 0);
#pragma unroll
                for (int t = 0; t < QT; ++t) tmem_ld_rows8(from + t * kSide, l[t]);
                if (with_key) {
#pragma unroll
                    for (int t = 0; t < QT; ++t) tmem_ld_rows8(from + Z::nq + t * kSide, c[t]);
                }
                const float2 f = *(const float2 *)&bars->factor[w.piece % kPieces][g * kGroup + 2 * q];
                const float2 scale[2] = {bars->scale[stage][t0], bars->scale[stage][t0 + 8]};
                tmem_wait_ld();
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const float sl = scale[d].x, sk = scale[d].y, log_sl = __log2f(sl);
                    per_sl[d] = exp2_fast(-log_sl);
                    auto term = [&](const uint32_t *x, int r) { return __uint_as_float(x[d * 2 + r]); };
                    float u0 = term(l[QT - 1], 0), u1 = term(l[QT - 1], 1), v0 = 0.f, v1 = 0.f;
#pragma unroll
                    for (int t = QT - 2; t >= 0; --t) fma2(u0, u1, u0, u1, 0.0625f, 0.0625f, term(l[t], 0), term(l[t], 1));
                    if (with_key) {
                        v0 = term(c[QT - 1], 0), v1 = term(c[QT - 1], 1);
#pragma unroll
                        for (int t = QT - 2; t >= 0; --t) fma2(v0, v1, v0, v1, 0.0625f, 0.0625f, term(c[t], 0), term(c[t], 1));
                        v0 *= sk, v1 *= sk;
                    }
                    fma2(u0, u1, u0, u1, sl, sl, v0, v1);
                    fma2(y[d][0], y[d][1], u0, u1, f.x, f.y, log_sl, log_sl);
                }
            }
            if (j0 + kTile > min(fewest, past)) {
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const int j = j0 + t0 + 8 * d;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (j >= past || j >= tokens - later[e]) y[d][e] = -INFINITY;
                }
                // cached rows that not all of the block's rows see, and those that came with the last ones, without NaN
                bar_test(smem_addr(&bars->full[stage]), round & 1);  // has completed: what the copy wrote is visible
                const int from = max(fewest - j0, 0), to = min((past - j0 + a.run - 1) / a.run * a.run, kTile);
#pragma unroll 1
                for (int k = from * 8 + threadIdx.x; k < to * 8; k += 128 * G)
#pragma unroll 1
                    for (int m = 0; m < tiles_m; ++m) {
                        uint4 *at = (uint4 *)(smem + stage * stage_bytes + m * kColBytes + k * 16);
                        const uint4 v = *at;
                        *at = make_uint4(without_nan(v.x), without_nan(v.y), without_nan(v.z), without_nan(v.w));
                    }
            }
            float x[2][2], most = -INFINITY;
#pragma unroll
            for (int d = 0; d < 2; ++d)
#pragma unroll
                for (int e = 0; e < 2; ++e) x[d][e] = y[d][e] + base[e], most = fmaxf(most, x[d][e]);
            if (group_any(g, most > kLimit)) {
                // a maximum anew, of the whole group's tokens
                float v[2], keep[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) v[e] = fmaxf(y[0][e], y[1][e]);
                join2(v, larger);
                if (lane < 4) *(float2 *)&bars->met[g][warp % 4][2 * q] = make_float2(v[0], v[1]);
                group_sync(g);
                float2 m = *(const float2 *)&bars->met[g][0][2 * q];
#pragma unroll
                for (int k = 1; k < 4; ++k) {
                    const float2 o = *(const float2 *)&bars->met[g][k][2 * q];
                    m.x = fmaxf(m.x, o.x), m.y = fmaxf(m.y, o.y);
                }
                const float high[2] = {m.x, m.y};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float anew = high[e] + base[e] > kLimit ? kRaise - high[e] : base[e];
                    keep[e] = anew == base[e] ? 1.f : exp2_fast(anew - base[e]);
                    base[e] = anew, sum[e] *= keep[e], x[0][e] = y[0][e] + anew, x[1][e] = y[1][e] + anew;
                }
                if (w.u > w.u0) {
                    if (warp % 4 == 0 && lane < 4) *(float2 *)&bars->keep[g][2 * q] = make_float2(keep[0], keep[1]);
                    group_sync(g);
                    pv_wait(i - 1);
                    tmem_after_sync();
                    float k[kGroup];
#pragma unroll
                    for (int r = 0; r < kGroup; r += 4) *(float4 *)(k + r) = *(const float4 *)&bars->keep[g][r];
#pragma unroll 1
                    for (int m = 0; m < tiles_m; ++m) {
                        uint32_t o[PT][kGroup];
#pragma unroll
                        for (int t = 0; t < PT; ++t) tmem_ld8(o_at + m * Z::np + t * kSide, o[t]);
                        tmem_wait_ld();
#pragma unroll
                        for (int t = 0; t < PT; ++t) {
#pragma unroll
                            for (int r = 0; r < kGroup; ++r) o[t][r] = __float_as_uint(__uint_as_float(o[t][r]) * k[r]);
                            tmem_st8(o_at + m * Z::np + t * kSide, o[t]);
                        }
                    }
                    tmem_wait_st();
                }
            }
            uint32_t h[2];
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const float p0 = exp2_fast(x[d][0]), p1 = exp2_fast(x[d][1]);
                fma2(sum[0], sum[1], p0, p1, per_sl[d], per_sl[d], sum[0], sum[1]);
                h[d] = pack2<__half>(p0, p1);
            }
            const uint32_t to = p_at + buffer * Z::p_bytes + g / 2 * PT * (kTile * 16) + t0 * 16 + side + 2 * q;
#pragma unroll
            for (int t = 0; t < PT; ++t)
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const uint32_t top = (h[d] + 0x00800080u) & 0xFF00FF00u;  // the upper byte, rounded
                    const __half2 rest = __hsub2(*(const __half2 *)&h[d], *(const __half2 *)&top);
                    *(__half2 *)&h[d] = __hmul2(rest, __floats2half2_rn(8.f, 8.f));
                    asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + t * (kTile * 16) + d * 128), "h"((uint16_t)__byte_perm(top, 0, 0x4431)) : "memory");
                }
            fence_async();
            tmem_before_sync();
            bar_arrive(smem_addr(&bars->p_ready[i & 1]));
            if (++stage == a.stages) stage = 0, ++round;
            if (++buffer == kWeights) buffer = 0;
            if (!w.last()) {
                w.next(a);
                continue;
            }
            // ------------------------------------------- the piece's end
            join2(sum, added);
            group_sync(g);  // what met before has been read
            if (lane < 4) *(float2 *)&bars->met[g][warp % 4][2 * q] = make_float2(sum[0], sum[1]);
            group_sync(g);
            const bool whole = w.u0 == 0 && w.u1 == w.n;
            // an unfinished piece: the part's last if it begins the request, else its first
            const int64_t slot = (int64_t)blockIdx.x * 2 + (w.u0 == 0);
            const int mine = min(kGroup, here - g * kGroup);
            if (warp % 4 == 0 && lane < 4) {
                // the rows' statistics; what their sums are multiplied with stays behind for the others
                float inv[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 2 * q + e;
                    const float all = (bars->met[g][0][r] + bars->met[g][1][r]) + (bars->met[g][2][r] + bars->met[g][3][r]);
                    inv[e] = all != 0.f ? 1.f / all : 0.f;
                    if (r < mine) {
                        if (!whole) a.stats[slot * R + g * kGroup + r] = make_float2(base[e], all);
                        else if (a.lse) a.lse[(int64_t)w.b * rows + rt * R + g * kGroup + r] = all != 0.f ? (log2f(all) - base[e]) * 0.6931471805599453f : -INFINITY;
                    }
                }
                *(float2 *)&bars->keep[g][2 * q] = make_float2(inv[0], inv[1]);
            }
            group_sync(g);
            float inv[kGroup];
#pragma unroll
            for (int j = 0; j < kGroup; j += 4) *(float4 *)(inv + j) = *(const float4 *)&bars->keep[g][j];
            pv_wait(i);
            tmem_after_sync();
            T *out = (T *)a.out + w.b * a.out_request;
            float *sums = a.sums + (slot * R + g * kGroup) * a.rank;
#pragma unroll 1
            for (int m = 0; m < tiles_m; ++m) {
                uint32_t o[PT][kGroup];
#pragma unroll
                for (int t = 0; t < PT; ++t) tmem_ld8(o_at + m * Z::np + t * kSide, o[t]);
                tmem_wait_ld();
                const int col = 128 * m + threadIdx.x % 128;
#pragma unroll
                for (int r = 0; r < kGroup; ++r) {
                    float v = __uint_as_float(o[PT - 1][r]);
#pragma unroll
                    for (int t = PT - 2; t >= 0; --t) v = fmaf(v, 0.125f, __uint_as_float(o[t][r]));
                    if (r < mine && col < a.rank) {
                        if (whole) out[bars->to[g * kGroup + r] + col] = elem<T>::from(inv[r] != 0.f ? v * inv[r] : 0.f);
                        else sums[(int64_t)r * a.rank + col] = v;
                    }
                }
            }
            tmem_before_sync();
            bar_arrive(smem_addr(&bars->o_free));
            w.next(a);
        }
    }
    __syncwarp();
    if (dead) bars->late = 1;
    tmem_before_sync();
    __syncthreads();
    if (bars->late) {  // a wait ran out somewhere: the block does not end while copies may be on their way (they take microseconds)
        for (int k = 0; k < 64; ++k) __nanosleep(100000);
    }
    if (warp == Z::soft) tmem_free(tmem, kCols);
}

// Joins the pieces of the requests that were cut, in the order of the parts,
// so that the result does not depend on timing.  Requests without a cached token
// get their zeros here.  WARPS warps share a row, each taking every WARPS-th piece.
constexpr int kJoinWarps = 8;

template <typename T, int R, int WARPS> __global__ void __launch_bounds__(kJoinWarps * 32) k_quantized_join(const __grid_constant__ Args a) {
    __shared__ float4 sum_of[WARPS > 1 ? kJoinWarps : 1][SIM_OP_MAX_RANK / 4];
    let_next_start();
    after_previous();  // the parts are written
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, mine = warp % WARPS;
    const int rows = a.new_tokens * a.heads;
    const int64_t row = (int64_t)blockIdx.x * (kJoinWarps / WARPS) + warp / WARPS;
    if (row >= (int64_t)a.requests * rows) return;
    const int b = (int)(row / rows), f = (int)(row - (int64_t)b * rows);
    const int tok = f / a.heads, h = f - tok * a.heads, rt = f / R, r = f % R;
    const int first = a.first[b], past = a.first[b + 1], total = a.first[a.requests];
    T *out = (T *)a.out + b * a.out_request + tok * a.out_token + h * a.out_head;
    if (first == past) {
        if (mine == 0) {
            for (int i = lane * 8; i < a.rank; i += 256) *(uint4 *)(out + i) = make_uint4(0, 0, 0, 0);
            if (a.lse && lane == 0) a.lse[row] = -INFINITY;
        }
        return;
    }
    // the parts that hold units [first, past)
    const int parts = parts_of(a, total);
    auto part_of = [&](int unit) { return (int)((((int64_t)unit + 1) * parts - 1) / total); };
    const int l0 = part_of(first + kRequestUnits), n = part_of(past - 1) - l0 + 1;
    if (n == 1) return;
    // piece l of the request: the last of its part where the request begins there, else the first
    auto slot = [&](int l) { return (((int64_t)(l0 + l) * a.row_tiles + rt) * 2 + (l == 0)) * R + r; };
    float m = -INFINITY;
    for (int l = lane; l < n; l += 32) m = fmaxf(m, -a.stats[slot(l)].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    float all = 0.f;
    float4 v[4] = {};
    for (int l1 = 0; l1 < n; l1 += 32) {
        const float2 st = l1 + lane < n ? a.stats[slot(l1 + lane)] : make_float2(kNothing, 0.f);
        const float w = l1 + lane < n ? exp2_fast(-st.x - m) : 0.f;
        all += warp_sum(w * st.y);
        const int k = min(32, n - l1);
#pragma unroll 4
        for (int l = mine; l < k; l += WARPS) {
            const float wl = __shfl_sync(~0u, w, l);
            const float *x = a.sums + slot(l1 + l) * a.rank + 4 * lane;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (128 * j + 4 * lane < a.rank) {
                    const float4 u = *(const float4 *)(x + 128 * j);
                    v[j].x += wl * u.x, v[j].y += wl * u.y, v[j].z += wl * u.z, v[j].w += wl * u.w;
                }
        }
    }
    if (WARPS > 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum_of[warp][lane + 32 * j] = v[j];
        __syncthreads();  // WARPS is the whole block: no warp of it has left
        if (mine) return;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            for (int k = 1; k < WARPS; ++k) {
                const float4 u = sum_of[k][lane + 32 * j];
                v[j].x += u.x, v[j].y += u.y, v[j].z += u.z, v[j].w += u.w;
            }
    }
    const float inv = all != 0.f ? 1.f / all : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (128 * j + 4 * lane < a.rank) {
            uint2 w = make_uint2(0, 0);
            if (all != 0.f) w = make_uint2(pack2<T>(v[j].x * inv, v[j].y * inv), pack2<T>(v[j].z * inv, v[j].w * inv));
            *(uint2 *)(out + 128 * j + 4 * lane) = w;
        }
    if (a.lse && lane == 0) a.lse[row] = all != 0.f ? (m + log2f(all)) * 0.6931471805599453f : -INFINITY;
}

// How the work is cut: row tiles side by side, and parts of the line of units.
struct Cut {
    int row_tiles, lanes;
    size_t first_bytes, sums_bytes, stats_bytes;
    size_t bytes() const { return first_bytes + sums_bytes + stats_bytes; }
};

Cut cut_for(int sms, int row_tile, int64_t requests, int64_t new_tokens, int64_t heads, int64_t rank) {
    Cut c;
    c.row_tiles = (int)((new_tokens * heads + row_tile - 1) / row_tile);
    c.lanes = c.row_tiles < sms ? sms / c.row_tiles : 1;
    const size_t parts = (size_t)c.row_tiles * c.lanes;
    c.first_bytes = ((size_t)(requests + 1) * 4 + 255) & ~(size_t)255;
    // one part has no unfinished pieces
    c.sums_bytes = c.lanes > 1 ? parts * 2 * row_tile * rank * 4 : 0;
    c.stats_bytes = c.lanes > 1 ? parts * 2 * row_tile * 8 : 0;
    return c;
}

// Rows of a block: 32 where there are so many and their sums and scores fit the tensor memory.
int row_tile_for(bool bf16, int64_t rows) { return bf16 && rows > kSide ? 2 * kSide : kSide; }

template <typename T, int G> int run(const Args &given, const CUtensorMap &map, const CUtensorMap &key, const Cut &c, cudaStream_t st) {
    using Z = Shape<T, G>;
    Args k = given;
    const int cols = (k.width + 127) / 128, steps = (k.width + 31) / 32;
    const int rest = 2 * steps * Z::chunk + kWeights * Z::p_bytes + (int)sizeof(Barriers<Z::rows>);
    k.stages = (kShared - rest) / (cols * kColBytes - (k.thin ? kColBytes / 2 : 0));
    if (k.stages > kMostStages) k.stages = kMostStages;
    static std::atomic<uint64_t> told;
    if (!allow_shared((const void *)k_quantized_decode<T, G>, kShared, told)) return SIM_ERR_CUDA;
    cudaError_t e = launch_early(k_quantized_decode<T, G>, c.row_tiles * c.lanes, Z::threads, kShared, 1, st, k, map, key);
    if (e != cudaSuccess) return launched("sim_op_quantized_decode", e);
    // few rows: a block shares the pieces of one; many: a warp has a row of its own
    const int64_t rows = (int64_t)k.requests * k.new_tokens * k.heads;
    const bool few = rows <= 1024;
    const int64_t per = few ? 1 : kJoinWarps;
    e = launch_early(few ? k_quantized_join<T, Z::rows, kJoinWarps> : k_quantized_join<T, Z::rows, 1>, (unsigned)((rows + per - 1) / per), kJoinWarps * 32, 0, 1, st, k);
    return launched("sim_op_quantized_decode (join)", e);
}

}  // namespace

unsigned quantized_faults() {
    unsigned n = 0;
    return cudaMemcpyFromSymbol(&n, g_faults, sizeof n) == cudaSuccess ? n : ~0u;
}

}  // namespace mtop

using namespace mtop;

extern "C" size_t sim_op_quantized_decode_workspace(int32_t requests, int32_t new_tokens, int32_t heads, int32_t rank) {
    if (requests < 1 || new_tokens < 1 || heads < 1 || rank < 1 || (int64_t)new_tokens * heads > INT32_MAX) return 256;
    const int sms = sm_count();
    if (!sms) return 0;
    const size_t x = cut_for(sms, kSide, requests, new_tokens, heads, rank).bytes(), y = cut_for(sms, 2 * kSide, requests, new_tokens, heads, rank).bytes();
    return x > y ? x : y;
}

extern "C" int sim_op_quantized_decode(const sim_op_quantized_decode_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16) return fail(SIM_ERR_ARG, "element type %d: 16-bit types only", a->type);
    if (a->requests < 0 || a->new_tokens < 0 || a->heads < 0 || a->blocks < 0 || a->table_blocks < 0)
        return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a->rank < 64 || a->rank > SIM_OP_MAX_RANK || a->rank % 64)
        return fail(SIM_ERR_ARG, "rank must be a multiple of 64 in [64, %d]", SIM_OP_MAX_RANK);
    if (a->key_dim < 0 || a->key_dim > SIM_OP_MAX_KEY || a->key_dim % 16)
        return fail(SIM_ERR_ARG, "key_dim must be a multiple of 16 in [0, %d]", SIM_OP_MAX_KEY);
    if (a->block_tokens < 1) return fail(SIM_ERR_ARG, "block_tokens must be at least 1");
    if (!std::isfinite(a->scale)) return fail(SIM_ERR_ARG, "scale must be finite");
    const int64_t rows = (int64_t)a->new_tokens * a->heads;
    if (rows == 0 || a->requests == 0) return SIM_OK;
    if (rows > INT32_MAX - 2 * kSide || a->requests * rows > INT32_MAX) return fail(SIM_ERR_ARG, "requests * new_tokens * heads must be below 2^31");
    if (!a->q || !a->out || !a->lengths || (!a->table && a->table_blocks) || ((!a->cache || !a->scales) && a->blocks))
        return fail(SIM_ERR_ARG, "q, cache, scales, table, lengths and out must not be NULL");
    if (!aligned16(a->q) || !aligned16(a->cache) || !aligned16(a->out) || !even_stride(a->requests, a->q_request) ||
        !even_stride(a->new_tokens, a->q_token) || !even_stride(a->heads, a->q_head) || !even_stride(a->requests, a->out_request) ||
        !even_stride(a->new_tokens, a->out_token) || !even_stride(a->heads, a->out_head))
        return fail(SIM_ERR_ARG, "q, cache and out must be aligned to 16 bytes, q and out with strides that are multiples of 8 elements");
    if ((a->blocks > 1 && a->cache_block % 16) || (a->block_tokens > 1 && a->cache_row % 16))
        return fail(SIM_ERR_ARG, "the cache's strides must be multiples of 16 elements");
    // the cache is one line of rows to the copies: a block must begin on one (blocks of one row are the rows)
    const int64_t cache_row = a->block_tokens > 1 ? a->cache_row : a->blocks > 1 && a->cache_block ? a->cache_block : a->rank + a->key_dim;
    if (cache_row < a->rank + a->key_dim || (a->blocks > 1 && (a->cache_block < 0 || a->cache_block % cache_row)))
        return fail(SIM_ERR_ARG, "cache_block must be a multiple of cache_row, which must hold a row");
    const int64_t ratio = a->blocks > 1 ? a->cache_block / cache_row : a->block_tokens, cache_rows = a->blocks ? (a->blocks - 1) * ratio + a->block_tokens : 0;
    if (cache_rows > INT32_MAX - 1 || ratio > INT32_MAX) return fail(SIM_ERR_ARG, "the cache must span fewer than 2^31 - 1 rows");
    const int64_t most = (int64_t)a->table_blocks * a->block_tokens;
    if (most > INT32_MAX - 65536) return fail(SIM_ERR_ARG, "table_blocks * block_tokens must be below 2^31 - 2^16");
    if (a->requests * (most / kUnit + 1 + kRequestUnits) > INT32_MAX) return fail(SIM_ERR_ARG, "requests * table_blocks * block_tokens is too large");
    if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < 256)
        return fail(SIM_ERR_ARG, "a workspace aligned to 256 bytes is needed");
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const bool bf = a->type == SIM_OP_BF16;
    const int row_tile = row_tile_for(bf, rows);
    const Cut c = cut_for(sms, row_tile, a->requests, a->new_tokens, a->heads, a->rank);
    if (a->workspace_bytes < c.bytes()) return fail(SIM_ERR_ARG, "the workspace must have %zu bytes", c.bytes());
    Args k;
    k.q = a->q, k.scales = a->scales, k.table = a->table, k.lengths = a->lengths, k.out = a->out, k.lse = a->lse;
    k.first = (int *)a->workspace;
    k.sums = (float *)((char *)a->workspace + c.first_bytes);
    k.stats = (float2 *)((char *)k.sums + c.sums_bytes);
    k.q_request = a->q_request, k.q_token = a->q_token, k.q_head = a->q_head;
    k.out_request = a->out_request, k.out_token = a->out_token, k.out_head = a->out_head, k.table_row = a->table_row;
    k.blocks = a->blocks, k.most = most;
    k.requests = a->requests, k.new_tokens = a->new_tokens, k.heads = a->heads, k.rank = a->rank, k.width = a->rank + a->key_dim;
    k.block_tokens = a->block_tokens, k.row_ratio = (int)ratio;
    k.row_tiles = c.row_tiles, k.lanes = c.lanes, k.none = (int)(cache_rows > 0 ? cache_rows : 1);
    k.scale_log2 = a->scale * 1.4426950408889634f;
    k.run = 4;
    while (k.run < kUnit && a->block_tokens % (2 * k.run) == 0) k.run *= 2;
    k.scattered = a->block_tokens % 4 != 0;
    // a key part that is the last column block alone takes half of it
    k.thin = a->rank % 128 == 0 && a->key_dim > 0;
    CUtensorMap map, key;
    const uint64_t size[2] = {(uint64_t)k.width, (uint64_t)k.none};
    const int64_t stride[1] = {a->blocks ? cache_row : k.width};
    const uint32_t box[2] = {128, k.scattered ? 1u : (uint32_t)k.run}, thin[2] = {64, box[1]};
    const void *cache = a->blocks ? a->cache : a->q;
    if (!byte_box_map(&map, cache, 2, size, stride, box) || !byte_box_map(&key, cache, 2, size, stride, thin)) return SIM_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    if (!bf) return run<__half, 2>(k, map, key, c, st);
    return row_tile == kSide ? run<__nv_bfloat16, 2>(k, map, key, c, st) : run<__nv_bfloat16, 4>(k, map, key, c, st);
}
