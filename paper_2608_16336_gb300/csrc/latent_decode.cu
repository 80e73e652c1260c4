// latent_decode.cu -- attention of new tokens over the block cache of latent
// vectors (mtsim_ops.h).
#include "tensor.cuh"

#include <cmath>

namespace mtop {
namespace {

// A block takes 64 rows (new token x head) of a request, over tiles of
// cached tokens:
//   S = Q C^T                 (64 x tile over the whole width)
//   P = exp2(S - m)
//   O += P C[:, :rank]        (64 x rank)
// A tile of C is one operand twice: rows are tokens for S, and for O the
// same bytes are read with the latent elements along the rows.  O fills the
// 512 columns of one half of the tensor memory's lanes (a product of 64 rows
// uses 16 of each 32), S the other half's first 128 columns, in two buffers, so
// that the scores of the next tile are computed while this tile's weights are.
//
// The tiles of all requests form one line, cut into equal parts, one a block
// (blocks of the same part and different rows run side by side, so that the
// second finds the cache rows in L2).  A part may begin and end inside
// a request: such pieces leave their sums in the workspace and k_join adds them.
//
// Bound by memory with one row tile: 3 requests of 90,001 to 130,000 tokens (406 MB)
// take 91.8 us, 4.4 TB/s, of which 20 us are start, end and join.  Bound by the
// chain from scores to sums with more: 64 requests of 200 to 10,240 tokens, 128
// heads take 105 us, 478 TFLOP/s (218 MB of cache would take 33 us to read).
constexpr int kRows = 64;
constexpr int kRowBlockBytes = kRows * 128;  // 64 rows of 64 elements
constexpr int kMaxBlocks = 9;                // 64-element column blocks of a row
constexpr int kSoftWarps = 4;
constexpr int kThreads = (kSoftWarps + 4) * 32;  // + products, cache copies, query copies (two)
constexpr int kMostStages = 8;
constexpr int kShared = 227 * 1024;  // Q, the stages, P, barriers

constexpr int kCols = 512;
constexpr uint32_t kHigh = operand_high(1024);
constexpr uint32_t kUpper = 16u << 16;  // the second 16 lanes of each 32

// Scores of 128 tokens and weights of 64 are held in buffers, tiles of the
// cache in as many stages as fit (Args::stages).
template <int TILE> struct Shape {
    static constexpr int scores = 128 / TILE, weights = 64 / TILE;
    static constexpr int block_bytes = TILE * 128;
};

struct Args {
    const void *q, *cache;
    const int32_t *table, *lengths;
    void *out;
    float *lse;
    int *first;      // [requests + 1]: the line's first tile of each request
    float *sums;     // [parts][2][64][rank]: the unfinished O of a part's first and last piece
    float2 *stats;   // [parts][2][64]: maximum and sum of weights
    int64_t q_request, q_token, q_head, out_request, out_token, out_head, cache_row, table_row;
    int64_t blocks, most;  // most: tokens a table can name
    int requests, new_tokens, heads, rank, width;
    int block_tokens, row_ratio;  // cache_block / cache_row
    int row_tiles, lanes;         // parts = row_tiles * lanes
    int tile;                     // tokens of a tile
    int stages;
    int q_pad;                    // rows of Q kept: 16, 32 or 64
    int run;                      // tokens a copy takes
    bool scattered;               // four rows anywhere instead of a run
    bool q_flat;                  // Q's rows are one line to the copies
    int none;                     // a row outside the cache
    float scale_log2;
    bool negative;
};

template <int TILE> struct Barriers {
    uint64_t full[kMostStages], empty[kMostStages][2], q_full, q_empty, s_ready[Shape<TILE>::scores];
    uint64_t p_ready[Shape<TILE>::weights], pv_done[Shape<TILE>::weights], o_free;
    uint32_t tmem;
    int first_request, first_tile, total;
    int spoiled[2];  // the last even and odd piece whose cached rows had infinities or NaN taken out
};

__device__ __forceinline__ int tokens_of(const Args &a, int b) {
    return (int)min(max((int64_t)a.lengths[b], (int64_t)0), a.most);
}
__device__ __forceinline__ int tiles_of(const Args &a, int b) { return (tokens_of(a, b) + a.tile - 1) / a.tile; }

// Parts in use (each has a tile at least) and where one begins on the line.
// As many parts as blocks and tiles allow; of few requests only so many that the
// join, whose time grows with the pieces of a row, does not outweigh the tiles
// saved (16 heads, 1 request of 8,000 tokens 22.0 us, with a part a block 26.0; of 3,000 17.8, 20.4).
__device__ __forceinline__ int parts_of(const Args &a, int total) {
    return max(1, min(a.lanes, min(total, (int)(5.f * __fsqrt_rn((float)total * a.requests)))));
}
__device__ __forceinline__ int begin_of(int total, int parts, int p) { return p < parts ? (int)((int64_t)total * p / parts) : total; }

// The pieces of a part: request b, tiles [t0, t1) of its n.
struct Piece {
    int b, t0, t1, n;
    int left;  // tiles of the part from t0 on
    __device__ bool start(const Args &a, int b0, int tile, int count) {
        b = b0, t0 = tile, left = count;
        return settle(a);
    }
    __device__ bool next(const Args &a) {
        left -= t1 - t0, ++b, t0 = 0;
        return b < a.requests && settle(a);
    }
    __device__ bool settle(const Args &a) {
        if (left <= 0) return false;
        n = tiles_of(a, b);
        while (n == 0) {  // tiles are left, so a request with some follows
            if (++b >= a.requests) return false;
            n = tiles_of(a, b);
        }
        t1 = min(n, t0 + left);
        return true;
    }
};

// Cached rows [from, to) of a tile that not all new tokens see.  A weight of
// 0 times infinity or NaN is not 0, so these become zeros (a thread takes 16 bytes of every second row),
template <typename T> __device__ __noinline__ void clean_rows(unsigned char *at, int from, int to) {
    for (int r = from + threadIdx.x / 64; r < to; r += 2) {
        uint4 &w = *(uint4 *)(at + r * 128);
        w = make_uint4(finite_only<T>(w.x), finite_only<T>(w.y), finite_only<T>(w.z), finite_only<T>(w.w));
    }
}
// and are added at the end to what the sums of the rows that see them have:
// tokens [j, past) of request b, of which this thread's two rows see those below see0 and see1.
template <typename T> __device__ __noinline__ void add_cleaned(const Args &a, int b, int j, int past, int see0, int see1, uint32_t o_at) {
    const int lane = threadIdx.x % 32;
    const int32_t *table = a.table + b * a.table_row;
    for (; j < past; ++j) {
        const int blk = j / a.block_tokens, id = table[blk];
        if (id < 0 || id >= a.blocks) continue;
        const T *row = (const T *)a.cache + ((int64_t)id * a.row_ratio + (j - blk * a.block_tokens)) * a.cache_row + 2 * (lane % 4);
        for (int c = 0; c < a.rank / 64; ++c, row += 64) {
            uint32_t o[32];
            tmem_ld_rows<64>(o_at + 64 * c, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float x = elem<T>::to(row[e / 2 * 8 + e % 2]);
                uint32_t &o0 = o[e / 2 * 4 + e % 2], &o1 = o[e / 2 * 4 + 2 + e % 2];
                if (!(fabsf(x) < INFINITY) && j < see0) o0 = __float_as_uint(__uint_as_float(o0) + x);
                if (!(fabsf(x) < INFINITY) && j < see1) o1 = __float_as_uint(__uint_as_float(o1) + x);
            }
            __syncwarp();
            tmem_st_rows64(o_at + 64 * c, o);
            tmem_wait_st();
        }
    }
}

// SEVERAL: calls of more than one new token (3 requests of 90,001 to 130,000 tokens, two
// new ones 92.0 us; without the two steps above 89.6, which calls of one do not pay).
template <typename T, int TILE, bool SEVERAL>
__global__ void __launch_bounds__(kThreads, 1) k_decode(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap m_cache, const __grid_constant__ CUtensorMap m_q) {
    using Z = Shape<TILE>;
    using R = WeightRange<T>;
    extern __shared__ __align__(1024) unsigned char smem[];
    // Q's column blocks hold only the rows there are (rounded up to 16, 32 or
    // 64): a product reads 64, and what it finds past them (the
    // following blocks, or the stages) makes rows that nothing looks at.
    const int blocks = (a.width + 63) / 64, q_block = a.q_pad * 128, stage_bytes = blocks * Z::block_bytes;
    const int stage_offset = blocks * q_block, p_offset = stage_offset + a.stages * stage_bytes;
    const uint32_t q_at = smem_addr(smem), stage_at = q_at + stage_offset, p_at = q_at + p_offset;
    Barriers<TILE> *bars = (Barriers<TILE> *)(smem + p_offset + kRowBlockBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rt = blockIdx.x % a.row_tiles, part = blockIdx.x / a.row_tiles;
    const int value_blocks = a.rank / 64, half = min(4, value_blocks);
    bool dead = false;
    let_next_start();

    if (warp == 1 && lane == 0) {
        for (int s = 0; s < a.stages; ++s) {
            bar_init(smem_addr(&bars->full[s]), 1);
            bar_init(smem_addr(&bars->empty[s][0]), 1);
            bar_init(smem_addr(&bars->empty[s][1]), 1);
        }
        bar_init(smem_addr(&bars->q_full), a.q_flat ? 1 : 64);
        bar_init(smem_addr(&bars->q_empty), 1);
        for (int s = 0; s < Z::scores; ++s) bar_init(smem_addr(&bars->s_ready[s]), 1);
        for (int s = 0; s < Z::weights; ++s) {
            bar_init(smem_addr(&bars->p_ready[s]), kSoftWarps * 32);
            bar_init(smem_addr(&bars->pv_done[s]), 1);
        }
        bar_init(smem_addr(&bars->o_free), kSoftWarps * 32);
        bars->spoiled[0] = bars->spoiled[1] = -1;
        bar_init_done();
    }
    if (warp == kSoftWarps) tmem_alloc(smem_addr(&bars->tmem), kCols);
    if (warp == kSoftWarps + 1 && lane == 0) fetch_map(&m_cache), fetch_map(&m_q);
    __syncwarp();
    after_previous();
    if (warp == 0) {
        // the line's length, and where this part begins on it; a lane keeps the
        // tiles of its first requests, so that most calls read the lengths once
        int total = 0, kept[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) kept[k] = 32 * k + lane < a.requests ? tiles_of(a, 32 * k + lane) : 0, total += kept[k];
        for (int b0 = 128; b0 < a.requests; b0 += 32) total += b0 + lane < a.requests ? tiles_of(a, b0 + lane) : 0;
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
            if (n && begin >= at && begin < at + n) bars->first_request = b0 + lane, bars->first_tile = begin - at;
            if (blockIdx.x == 0 && b0 + lane < a.requests) a.first[b0 + lane] = at;
            seen += __shfl_sync(~0u, incl, 31);
        };
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (32 * k < a.requests) place(32 * k, kept[k]);
        for (int b0 = 128; b0 < a.requests; b0 += 32) place(b0, b0 + lane < a.requests ? tiles_of(a, b0 + lane) : 0);
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
    Piece pc;
    bool more = pc.start(a, end > begin ? bars->first_request : 0, end > begin ? bars->first_tile : 0, end - begin);

    if (warp == kSoftWarps + 1) {
        // ----------------------------------------------------- cache copies
        // a copy takes `run` tokens of a block by one column block, or, where
        // blocks are not whole multiples of 4 tokens, any four rows
        const int run = a.run, groups = TILE / run, group = lane % groups, c0 = lane / groups, step = 32 / groups;
        int s = 0;
        uint32_t round = 0;
        for (; more; more = pc.next(a)) {
            const int tokens = tokens_of(a, pc.b);
            const int32_t *table = a.table + pc.b * a.table_row;
            for (int t = pc.t0; t < pc.t1; ++t) {
                int row[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = t * TILE + run * group + e;
                    row[e] = a.none;
                    if ((e == 0 || a.scattered) && j < tokens) {
                        const int blk = j / a.block_tokens, id = table[blk];
                        if (id >= 0 && id < a.blocks) row[e] = id * a.row_ratio + (j - blk * a.block_tokens);
                    }
                }
                const uint32_t parity = (round & 1) ^ 1, full = smem_addr(&bars->full[s]);
                const uint32_t dst = stage_at + s * stage_bytes + group * run * 128;
                auto copy = [&](int c) {
                    if (a.scattered) copy_rows_4(dst + c * Z::block_bytes, &m_cache, 64 * c, row[0], row[1], row[2], row[3], full);
                    else copy_box_2d(dst + c * Z::block_bytes, &m_cache, 64 * c, row[0], full);
                };
                bar_wait(smem_addr(&bars->empty[s][0]), parity, dead);
                if (lane == 0) bar_expect(full, blocks * Z::block_bytes);
                __syncwarp();
                int c = c0;
                for (; c < half; c += step) copy(c);
                bar_wait(smem_addr(&bars->empty[s][1]), parity, dead);
                for (; c < blocks; c += step) copy(c);
                if (++s == a.stages) s = 0, ++round;
            }
        }
    } else if (warp >= kSoftWarps + 2 && a.q_flat) {
        // ----------------------------------------------------- query copies
        for (int k = 0; more && warp == kSoftWarps + 2 && lane == 0; more = pc.next(a), ++k) {
            const uint32_t full = smem_addr(&bars->q_full);
            bar_wait(smem_addr(&bars->q_empty), (k & 1) ^ 1, dead);
            bar_expect(full, blocks * q_block);
            for (int c = 0; c < blocks; ++c) copy_box_3d(q_at + c * q_block, &m_q, 64 * c, rt * kRows, pc.b, full);
        }
    } else if (warp >= kSoftWarps + 2) {
        // the same for queries whose (token, head) rows are not evenly spaced:
        // eight lanes a row of 128 bytes; the two warps take every second group of four rows
        const int r0 = (warp - kSoftWarps - 2) * 4 + lane / 8, col = 8 * (lane % 8), n = a.q_pad / 8;
        int64_t from[8];
        uint32_t dst[8], real = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int r = r0 + 8 * k, flat = rt * kRows + r, tok = flat / a.heads, h = flat - tok * a.heads;
            if (tok < a.new_tokens) real |= 1u << k;
            from[k] = tok < a.new_tokens ? tok * a.q_token + h * a.q_head + col : 0;
            dst[k] = q_at + r * 128 + (((lane % 8) ^ (r & 7)) << 4);
        }
        for (int k = 0; more; more = pc.next(a), ++k) {
            bar_wait(smem_addr(&bars->q_empty), (k & 1) ^ 1, dead);
            const T *q = (const T *)a.q + pc.b * a.q_request;
#pragma unroll
            for (int c = 0; c < kMaxBlocks; ++c)
                if (c < blocks) {
                    const bool in = col + 64 * c < a.width;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < n) {
                            const bool copy = in && (real >> e & 1);
                            copy_16(dst[e] + c * q_block, copy ? q + from[e] + 64 * c : (const T *)a.q, copy);
                        }
                }
            copy_16_done();
            fence_async();
            bar_arrive(smem_addr(&bars->q_full));
        }
    } else if (warp == kSoftWarps) {
        // -------------------------------------------------------- products
        const bool bf = std::is_same<T, __nv_bfloat16>::value;
        const uint32_t word_s = product_word(kRows, TILE, bf, false, a.negative);
        auto scores = [&](int i, int s) {
            const uint32_t d = tmem + kUpper + i % Z::scores * TILE;
            uint32_t q_low = operand_low(q_at, 16), c_low = operand_low(stage_at + s * stage_bytes, 16);
            for (int c = 0; c < blocks; ++c, q_low += q_block >> 4, c_low += Z::block_bytes >> 4)
#pragma unroll
                for (int k = 0; k < 4; ++k) product_ss<kHigh, kHigh>(d, q_low + 2 * k, c_low + 2 * k, word_s, c + k > 0);
            product_commit(smem_addr(&bars->s_ready[i % Z::scores]));
        };
        auto weighted = [&](int i, int s, bool add) {
            const int w = i % Z::weights;
            const uint32_t w_low = operand_low(p_at + w * (TILE * 2), 16);
            uint32_t c_low = operand_low(stage_at + s * stage_bytes, Z::block_bytes);
            for (int c = 0; c < value_blocks; c += 4, c_low += 4 * Z::block_bytes >> 4) {
                const uint32_t word = product_word(kRows, 64 * min(4, value_blocks - c), bf, true, false);
#pragma unroll
                for (int e = 0; e < TILE / 16; ++e)
                    product_ss<kHigh, kHigh>(tmem + 64 * c, w_low + 2 * e, c_low + 128 * e, word, add || e > 0);
                if (c == 0) product_commit(smem_addr(&bars->empty[s][0]));
            }
            product_commit(smem_addr(&bars->empty[s][1]));
            product_commit(smem_addr(&bars->pv_done[w]));
        };
        // Scores run ahead of the weighted sums by as many tiles as there are
        // buffers; whichever can go goes, so that neither waits for the other's
        // operands.  One thread does it all.
        const int n = end - begin;
        Piece ps = pc;                // where the scores are: tile ts of piece ps
        int si = 0, wi = 0, ks = 0, kw = 0, s_stage = 0, w_stage = 0;
        uint32_t s_round = 0;
        int ts = pc.t0, tw = pc.t0;
        bool q_here = false;
        const bool elected = elect_one();
        for (int idle = 0; elected && wi < n && more && idle < kPollLimit && !dead;) {
            bool went = false;
            if (si < n && si - wi < Z::scores) {
                if (!q_here) q_here = bar_poll(smem_addr(&bars->q_full), ks & 1);
                if (q_here && bar_poll(smem_addr(&bars->full[s_stage]), s_round & 1)) {
                    tmem_after_sync();
                    scores(si, s_stage);
                    ++si, went = true;
                    if (++s_stage == a.stages) s_stage = 0, ++s_round;
                    if (++ts == ps.t1) {
                        product_commit(smem_addr(&bars->q_empty));
                        q_here = false, ++ks;
                        if (si < n && ps.next(a)) ts = ps.t0;
                    }
                }
            }
            if (wi < si && bar_poll(smem_addr(&bars->p_ready[wi % Z::weights]), (wi / Z::weights) & 1)) {
                if (tw == pc.t0 && kw > 0) bar_wait(smem_addr(&bars->o_free), (kw - 1) & 1, dead);
                tmem_after_sync();
                weighted(wi, w_stage, tw > pc.t0);
                ++wi, went = true;
                if (++w_stage == a.stages) w_stage = 0;
                if (++tw == pc.t1) {
                    ++kw, more = pc.next(a);
                    tw = pc.t0;
                }
            }
            idle = went ? 0 : idle + 1;
            if (idle == kPollLimit) atomicAdd(&g_faults, 1u);
        }
        __syncwarp();
    } else if (warp < kSoftWarps) {
        // ------------------------------------------------- weights and sums
        const uint32_t lanes = (uint32_t)warp << 21;
        const uint32_t s_at = tmem + kUpper + lanes, o_at = tmem + lanes;
        const int r0 = warp * 16 + lane / 4;  // this thread's rows: r0 and r0 + 8
        int see0 = 0, see1 = 0;
        const int f0 = rt * kRows + r0, f1 = f0 + 8;
        const int tok0 = f0 / a.heads, tok1 = f1 / a.heads;
        const bool real0 = tok0 < a.new_tokens, real1 = tok1 < a.new_tokens;
        // where P goes: row r, 16-byte chunk (k ^ r % 8), 4 bytes of it
        const uint32_t p0 = p_at + r0 * 128 + (lane % 4) * 4, p1 = p0 + 8 * 128;
        const int swz = r0 & 7;
        // the rows this lane writes out at the end of a piece, 16 bytes of each
        int64_t to[4];
        uint32_t leaves = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int flat = rt * kRows + warp * 16 + 4 * k + lane / 8, tok = flat / a.heads;
            if (tok < a.new_tokens) leaves |= 1u << k;
            to[k] = tok * a.out_token + (flat - tok * a.heads) * a.out_head + 8 * (lane % 8);
        }
        int i = 0, stage_of = 0;
        for (int k = 0; more; more = pc.next(a), ++k) {
            const int tokens = tokens_of(a, pc.b);
            see0 = tokens - a.new_tokens + 1 + min(tok0, a.new_tokens - 1);
            see1 = tokens - a.new_tokens + 1 + min(tok1, a.new_tokens - 1);
            const int fewest = tokens - a.new_tokens + 1;
            float top0 = -INFINITY, top1 = -INFINITY, sum0 = 0.f, sum1 = 0.f;
            for (int t = pc.t0; t < pc.t1; ++t, ++i, stage_of = stage_of + 1 == a.stages ? 0 : stage_of + 1) {
                bar_wait(smem_addr(&bars->s_ready[i % Z::scores]), (i / Z::scores) & 1, dead);
                tmem_after_sync();
                uint32_t s[TILE / 2];
                float *x = (float *)s;
                tmem_ld_rows<TILE>(s_at + i % Z::scores * TILE, s);
                tmem_wait_ld();
                if ((t + 1) * TILE > tokens && !a.scattered) {
                    // rows past the request's tokens came with their block and may hold anything: zeros, as 0 * NaN is NaN
                    const int from = tokens - t * TILE;
                    unsigned char *stage = smem + stage_offset + stage_of * stage_bytes;
                    for (int c = 0; c < value_blocks; ++c)
                        for (int e = from * 8 + threadIdx.x; e < TILE * 8; e += kSoftWarps * 32)
                            *(uint4 *)(stage + c * Z::block_bytes + e * 16) = make_uint4(0, 0, 0, 0);
                }
                if (SEVERAL && (t + 1) * TILE > fewest) {
                    // (little code: it runs once a request, and fetching it is what it costs)
                    bar_test(smem_addr(&bars->full[stage_of]), (i / a.stages) & 1);  // has completed: what the copy wrote is visible
                    const int c = threadIdx.x / 8 % 8, from = max(fewest - t * TILE, 0), to = c < value_blocks ? min(tokens - t * TILE, TILE) : 0;
                    unsigned char *at = smem + stage_offset + stage_of * stage_bytes + c * Z::block_bytes + threadIdx.x % 8 * 16;
                    uint32_t sum = 0;
#pragma unroll 1
                    for (int r = from + threadIdx.x / 64; r < to; r += 2) {
                        const uint4 w = *(const uint4 *)(at + r * 128);
                        spoil<T>(sum, w.x), spoil<T>(sum, w.y), spoil<T>(sum, w.z), spoil<T>(sum, w.w);
                    }
                    if (spoiled(sum)) clean_rows<T>(at, from, to), bars->spoiled[k & 1] = k;
                    __syncwarp();
                }
                if ((t + 1) * TILE > fewest) {
                    const int c0 = t * TILE + 2 * (lane % 4);
#pragma unroll
                    for (int e = 0; e < TILE / 8; ++e)
#pragma unroll
                        for (int d = 0; d < 2; ++d) {
                            if (c0 + 8 * e + d >= see0) x[4 * e + d] = -INFINITY;
                            if (c0 + 8 * e + d >= see1) x[4 * e + 2 + d] = -INFINITY;
                        }
                }
                float m0 = fmaxf(x[0], x[1]), m1 = fmaxf(x[2], x[3]);
#pragma unroll
                for (int e = 1; e < TILE / 8; ++e) {
                    m0 = fmaxf(m0, fmaxf(x[4 * e], x[4 * e + 1]));
                    m1 = fmaxf(m1, fmaxf(x[4 * e + 2], x[4 * e + 3]));
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    m0 = fmaxf(m0, __shfl_xor_sync(~0u, m0, o));
                    m1 = fmaxf(m1, __shfl_xor_sync(~0u, m1, o));
                }
                const float high0 = real0 ? m0 * a.scale_log2 : -INFINITY, high1 = real1 ? m1 * a.scale_log2 : -INFINITY;
                // sums are rescaled only when the maximum has grown by 2^grow: weights up to that are as exact
                const bool grow0 = high0 > top0 + R::grow || (top0 == -INFINITY && high0 > -INFINITY);
                const bool grow1 = high1 > top1 + R::grow || (top1 == -INFINITY && high1 > -INFINITY);
                float keep0 = 1.f, keep1 = 1.f;
                if (grow0) keep0 = top0 == -INFINITY ? 0.f : exp2_fast(top0 - high0), top0 = high0;
                if (grow1) keep1 = top1 == -INFINITY ? 0.f : exp2_fast(top1 - high1), top1 = high1;
                sum0 *= keep0, sum1 *= keep1;
                float base0 = top0 == -INFINITY ? 0.f : R::raise - top0, base1 = top1 == -INFINITY ? 0.f : R::raise - top1;
                float by = a.scale_log2;
                // (a row that is infinite or NaN leaves its neighbours' rounding as it is)
                if (__any_sync(~0u, (beyond_fused(top0) && fabsf(top0) < INFINITY) || (beyond_fused(top1) && fabsf(top1) < INFINITY))) {
                    by = 1.f, base0 = base1 = R::raise;
#pragma unroll
                    for (int e = 0; e < TILE / 2; ++e) x[e] = below_top(x[e], a.scale_log2, e & 2 ? top1 : top0);
                }
                uint32_t p[TILE / 4];
#pragma unroll
                for (int e = 0; e < TILE / 8; ++e) {
                    float a0, a1, b0, b1;
                    fma2(a0, a1, x[4 * e], x[4 * e + 1], by, by, base0, base0);
                    fma2(b0, b1, x[4 * e + 2], x[4 * e + 3], by, by, base1, base1);
                    a0 = exp2_fast(a0), a1 = exp2_fast(a1), b0 = exp2_fast(b0), b1 = exp2_fast(b1);
                    sum0 += a0 + a1, sum1 += b0 + b1;
                    p[2 * e] = pack2<T>(a0, a1), p[2 * e + 1] = pack2<T>(b0, b1);
                }
                // P's buffer has been read; before a rescaling, O is at rest too
                auto wait_pv = [&](int j) { bar_wait(smem_addr(&bars->pv_done[j % Z::weights]), (j / Z::weights) & 1, dead); };
                if (i >= Z::weights) wait_pv(i - Z::weights);
                if (t > pc.t0 && __any_sync(~0u, grow0 || grow1)) {
                    wait_pv(i - 1);
                    tmem_after_sync();
                    for (int c = 0; c < value_blocks; ++c) {
                        uint32_t o[32];
                        tmem_ld_rows<64>(o_at + 64 * c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            o[e] = __float_as_uint(__uint_as_float(o[e]) * keep0);
                            o[e + 1] = __float_as_uint(__uint_as_float(o[e + 1]) * keep0);
                            o[e + 2] = __float_as_uint(__uint_as_float(o[e + 2]) * keep1);
                            o[e + 3] = __float_as_uint(__uint_as_float(o[e + 3]) * keep1);
                        }
                        tmem_st_rows64(o_at + 64 * c, o);
                    }
                    tmem_wait_st();
                }
#pragma unroll
                for (int e = 0; e < TILE / 8; ++e) {
                    const uint32_t chunk = (uint32_t)(((e + i % Z::weights * (TILE / 8)) ^ swz) << 4);
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(p0 + chunk), "r"(p[2 * e]) : "memory");
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(p1 + chunk), "r"(p[2 * e + 1]) : "memory");
                }
                fence_async();
                tmem_before_sync();
                bar_arrive(smem_addr(&bars->p_ready[i % Z::weights]));
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                sum0 += __shfl_xor_sync(~0u, sum0, o);
                sum1 += __shfl_xor_sync(~0u, sum1, o);
            }
            bar_wait(smem_addr(&bars->pv_done[(i - 1) % Z::weights]), ((i - 1) / Z::weights) & 1, dead);
            tmem_after_sync();
            const bool whole = pc.t0 == 0 && pc.t1 == pc.n;
            // an unfinished piece: the part's last if it begins the request, else its first
            const int64_t slot = (int64_t)blockIdx.x * 2 + (pc.t0 == 0);
            // (a sum of 0 is a row that sees nothing: zeros; one that is no number stays so)
            const float inv0 = sum0 != 0.f ? 1.f / sum0 : 0.f, inv1 = sum1 != 0.f ? 1.f / sum1 : 0.f;
            float *sums = a.sums + (slot * kRows + warp * 16) * a.rank;
            T *out = (T *)a.out + pc.b * a.out_request;
            if (SEVERAL && pc.t1 * TILE > fewest) {
                asm volatile("bar.sync 1, %0;" ::"n"(kSoftWarps * 32) : "memory");  // all have said whether there were some
                if (*(volatile int *)&bars->spoiled[k & 1] == k) add_cleaned<T>(a, pc.b, max(fewest, pc.t0 * TILE), min(tokens, pc.t1 * TILE), see0, see1, o_at);
            }
            // Fragments hold 8 bytes of a row; through the (now idle) rows of P
            // they leave as 128 bytes of a row.  A warp has 16 rows of its own there.
            for (int c = 0; c < value_blocks; ++c) {
                uint32_t o[32];
                float *v = (float *)o;
                tmem_ld_rows<64>(o_at + 64 * c, o);
                tmem_wait_ld();
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t chunk = (uint32_t)((e ^ swz) << 4);
                        const uint32_t w0 = sum0 != 0.f ? pack2<T>(v[4 * e] * inv0, v[4 * e + 1] * inv0) : 0u;
                        const uint32_t w1 = sum1 != 0.f ? pack2<T>(v[4 * e + 2] * inv1, v[4 * e + 3] * inv1) : 0u;
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(p0 + chunk), "r"(w0) : "memory");
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(p1 + chunk), "r"(w1) : "memory");
                    }
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = 4 * k + lane / 8;
                        const uint4 w = *(const uint4 *)(smem + p_offset + (warp * 16 + r) * 128 + (((lane % 8) ^ (r & 7)) << 4));
                        if (leaves >> k & 1) *(uint4 *)(out + to[k] + 64 * c) = w;
                    }
                    __syncwarp();
                } else {
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int turn = (r0 & 3) << 1 | (r0 >> 2 & 1);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t at = (uint32_t)(((2 * e + (lane % 4) / 2) ^ turn) << 4 | (lane & 1) << 3);
                            const float *x = v + 16 * hf + 4 * e;
                            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(p_at + r0 * 128 + at), "f"(x[0]), "f"(x[1]) : "memory");
                            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(p_at + (r0 + 8) * 128 + at), "f"(x[2]), "f"(x[3]) : "memory");
                        }
                        __syncwarp();
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int r = 4 * k + lane / 8, tr = (r & 3) << 1 | (r >> 2 & 1);
                            const uint4 w = *(const uint4 *)(smem + p_offset + (warp * 16 + r) * 128 + (((lane % 8) ^ tr) << 4));
                            if (leaves >> k & 1) *(uint4 *)(sums + r * a.rank + 64 * c + 32 * hf + 4 * (lane % 8)) = w;
                        }
                        __syncwarp();
                    }
                }
            }
            tmem_before_sync();
            bar_arrive(smem_addr(&bars->o_free));
            if (lane % 4 == 0) {
                if (whole) {
                    const int64_t at = (int64_t)pc.b * a.new_tokens * a.heads;
                    if (real0 && a.lse) a.lse[at + f0] = sum0 != 0.f ? (top0 + (log2f(sum0) - R::raise)) * 0.6931471805599453f : -INFINITY;
                    if (real1 && a.lse) a.lse[at + f1] = sum1 != 0.f ? (top1 + (log2f(sum1) - R::raise)) * 0.6931471805599453f : -INFINITY;
                } else {
                    a.stats[slot * kRows + r0] = make_float2(top0, sum0);
                    a.stats[slot * kRows + r0 + 8] = make_float2(top1, sum1);
                }
            }
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    if (warp == kSoftWarps) tmem_free(tmem, kCols);
}

// Joins the pieces of the requests that were cut, in the order of the parts,
// so that the result does not depend on timing.  Requests without a cached token
// get their zeros here.  WARPS warps share a row, each taking every WARPS-th piece.
constexpr int kJoinWarps = 8;

template <typename T, int WARPS> __global__ void __launch_bounds__(kJoinWarps * 32) k_join(const __grid_constant__ Args a) {
    __shared__ float4 sum_of[WARPS > 1 ? kJoinWarps : 1][SIM_OP_MAX_RANK / 4];
    let_next_start();
    after_previous();  // the parts are written
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, mine = warp % WARPS;
    const int rows = a.new_tokens * a.heads;
    const int64_t row = (int64_t)blockIdx.x * (kJoinWarps / WARPS) + warp / WARPS;
    if (row >= (int64_t)a.requests * rows) return;
    const int b = (int)(row / rows), f = (int)(row - (int64_t)b * rows);
    const int tok = f / a.heads, h = f - tok * a.heads, rt = f / kRows, r = f % kRows;
    const int first = a.first[b], past = a.first[b + 1], total = a.first[a.requests];
    T *out = (T *)a.out + b * a.out_request + tok * a.out_token + h * a.out_head;
    if (first == past) {
        if (mine == 0) {
            for (int i = lane * 8; i < a.rank; i += 256) *(uint4 *)(out + i) = make_uint4(0, 0, 0, 0);
            if (a.lse && lane == 0) a.lse[row] = -INFINITY;
        }
        return;
    }
    // the parts that hold tiles [first, past)
    const int parts = parts_of(a, total);
    auto part_of = [&](int tile) { return (int)((((int64_t)tile + 1) * parts - 1) / total); };
    const int l0 = part_of(first), n = part_of(past - 1) - l0 + 1;
    if (n == 1) return;
    // piece l of the request: the last of its part where the request begins there, else the first
    auto slot = [&](int l) { return (((int64_t)(l0 + l) * a.row_tiles + rt) * 2 + (l == 0)) * kRows + r; };
    float m = -INFINITY;
    for (int l = lane; l < n; l += 32) m = fmaxf(m, a.stats[slot(l)].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    float all = 0.f;
    float4 v[4] = {};
    for (int l1 = 0; l1 < n; l1 += 32) {
        const float2 st = l1 + lane < n ? a.stats[slot(l1 + lane)] : make_float2(-INFINITY, 0.f);
        const float w = st.x == -INFINITY ? 0.f : exp2_fast(st.x - m);
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
    if (a.lse && lane == 0) a.lse[row] = all != 0.f ? (m + (log2f(all) - WeightRange<T>::raise)) * 0.6931471805599453f : -INFINITY;
}

// How the work is cut: row tiles side by side, and parts of the line of tiles.
struct Cut {
    int row_tiles, lanes;
    size_t first_bytes, sums_bytes, stats_bytes;
    size_t bytes() const { return first_bytes + sums_bytes + stats_bytes; }
};

Cut cut_for(int sms, int64_t requests, int64_t new_tokens, int64_t heads, int64_t rank) {
    Cut c;
    c.row_tiles = (int)((new_tokens * heads + kRows - 1) / kRows);
    c.lanes = c.row_tiles < sms ? sms / c.row_tiles : 1;
    const size_t parts = (size_t)c.row_tiles * c.lanes;
    c.first_bytes = ((size_t)(requests + 1) * 4 + 255) & ~(size_t)255;
    // one part has no unfinished pieces
    c.sums_bytes = c.lanes > 1 ? parts * 2 * kRows * rank * 4 : 0;
    c.stats_bytes = c.lanes > 1 ? parts * 2 * kRows * 8 : 0;
    return c;
}

template <typename T> int run(const Args &k, const CUtensorMap &m_cache, const CUtensorMap &m_q, const Cut &c, cudaStream_t st) {
    const bool several = k.new_tokens > 1;
    auto kernel = k.tile == 32 ? (several ? k_decode<T, 32, true> : k_decode<T, 32, false>) : several ? k_decode<T, 64, true> : k_decode<T, 64, false>;
    static std::atomic<uint64_t> told[4];
    if (!allow_shared((const void *)kernel, kShared, told[2 * (k.tile == 32) + several])) return SIM_ERR_CUDA;
    cudaError_t e = launch_early(kernel, c.row_tiles * c.lanes, kThreads, kShared, 1, st, k, m_cache, m_q);
    if (e != cudaSuccess) return launched("sim_op_latent_decode", e);
    // Few rows: a block shares the pieces of one; many: a warp has a row of its
    // own.  2 x 128 heads 27.2 us (a warp a row 54.7), 8 x 128 31.8 (45.0), 64 x 16 59.6
    // (59.9); a warp a row for 16 x 128 heads 49.7 (a block 50.1), 64 x 128 100 (127).
    const int64_t rows = (int64_t)k.requests * k.new_tokens * k.heads;
    const bool few = rows <= 1024;
    const int64_t per = few ? 1 : kJoinWarps;
    e = launch_early(few ? k_join<T, kJoinWarps> : k_join<T, 1>, (unsigned)((rows + per - 1) / per), kJoinWarps * 32, 0, 1, st, k);
    return launched("sim_op_latent_decode (join)", e);
}

}  // namespace

unsigned decode_faults() {
    unsigned n = 0;
    return cudaMemcpyFromSymbol(&n, g_faults, sizeof n) == cudaSuccess ? n : ~0u;
}

}  // namespace mtop

using namespace mtop;

extern "C" size_t sim_op_latent_decode_workspace(int32_t requests, int32_t new_tokens, int32_t heads, int32_t rank) {
    if (requests < 1 || new_tokens < 1 || heads < 1 || rank < 1 || (int64_t)new_tokens * heads > INT32_MAX) return 256;
    const int sms = sm_count();
    return sms ? cut_for(sms, requests, new_tokens, heads, rank).bytes() : 0;
}

extern "C" int sim_op_latent_decode(const sim_op_latent_decode_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16) return fail(SIM_ERR_ARG, "element type %d: 16-bit types only", a->type);
    if (a->requests < 0 || a->new_tokens < 0 || a->heads < 0 || a->blocks < 0 || a->table_blocks < 0)
        return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a->rank < 64 || a->rank > SIM_OP_MAX_RANK || a->rank % 64)
        return fail(SIM_ERR_ARG, "rank must be a multiple of 64 in [64, %d]", SIM_OP_MAX_RANK);
    if (a->key_dim < 0 || a->key_dim > SIM_OP_MAX_KEY || a->key_dim % 8)
        return fail(SIM_ERR_ARG, "key_dim must be a multiple of 8 in [0, %d]", SIM_OP_MAX_KEY);
    if (a->block_tokens < 1) return fail(SIM_ERR_ARG, "block_tokens must be at least 1");
    if (!std::isfinite(a->scale)) return fail(SIM_ERR_ARG, "scale must be finite");
    const int64_t rows = (int64_t)a->requests * a->new_tokens * a->heads;
    if (rows == 0) return SIM_OK;
    if (rows > INT32_MAX) return fail(SIM_ERR_ARG, "requests * new_tokens * heads must be below 2^31");
    if (!a->q || !a->out || !a->lengths || (!a->table && a->table_blocks) || (!a->cache && a->blocks))
        return fail(SIM_ERR_ARG, "q, cache, table, lengths and out must not be NULL");
    if (!aligned16(a->q) || !aligned16(a->cache) || !aligned16(a->out) || !even_stride(a->requests, a->q_request) ||
        !even_stride(a->new_tokens, a->q_token) || !even_stride(a->heads, a->q_head) || !even_stride(a->blocks, a->cache_block) ||
        !even_stride(a->block_tokens, a->cache_row) || !even_stride(a->requests, a->out_request) ||
        !even_stride(a->new_tokens, a->out_token) || !even_stride(a->heads, a->out_head))
        return fail(SIM_ERR_ARG, "q, cache and out must be aligned to 16 bytes, with strides that are multiples of 8 elements");
    // the cache is one line of rows to the copies: a block must begin on one (blocks of one row are the rows)
    const int64_t cache_row = a->block_tokens > 1 ? a->cache_row : a->blocks > 1 && a->cache_block ? a->cache_block : a->rank + a->key_dim;
    if (cache_row < a->rank + a->key_dim || (a->blocks > 1 && (a->cache_block < 0 || a->cache_block % cache_row)))
        return fail(SIM_ERR_ARG, "cache_block must be a multiple of cache_row, which must hold a row");
    const int64_t ratio = a->blocks > 1 ? a->cache_block / cache_row : a->block_tokens, cache_rows = a->blocks ? (a->blocks - 1) * ratio + a->block_tokens : 0;
    if (cache_rows > INT32_MAX - 1 || ratio > INT32_MAX) return fail(SIM_ERR_ARG, "the cache must span fewer than 2^31 - 1 rows");
    const int64_t most = (int64_t)a->table_blocks * a->block_tokens;
    if (most > INT32_MAX - 65536) return fail(SIM_ERR_ARG, "table_blocks * block_tokens must be below 2^31 - 2^16");
    if (a->requests * (most / 32 + 1) > INT32_MAX) return fail(SIM_ERR_ARG, "requests * table_blocks * block_tokens is too large");
    if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < 256)
        return fail(SIM_ERR_ARG, "a workspace aligned to 256 bytes is needed");
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    const Cut c = cut_for(sms, a->requests, a->new_tokens, a->heads, a->rank);
    if (a->workspace_bytes < c.bytes()) return fail(SIM_ERR_ARG, "the workspace must have %zu bytes", c.bytes());
    Args k;
    k.q = a->q, k.cache = a->cache, k.table = a->table, k.lengths = a->lengths, k.out = a->out, k.lse = a->lse;
    k.first = (int *)a->workspace;
    k.sums = (float *)((char *)a->workspace + c.first_bytes);
    k.stats = (float2 *)((char *)k.sums + c.sums_bytes);
    k.q_request = a->q_request, k.q_token = a->q_token, k.q_head = a->q_head;
    k.out_request = a->out_request, k.out_token = a->out_token, k.out_head = a->out_head, k.cache_row = cache_row, k.table_row = a->table_row;
    k.blocks = a->blocks, k.most = most;
    k.requests = a->requests, k.new_tokens = a->new_tokens, k.heads = a->heads, k.rank = a->rank, k.width = a->rank + a->key_dim;
    k.block_tokens = a->block_tokens, k.row_ratio = (int)ratio;
    k.row_tiles = c.row_tiles, k.lanes = c.lanes, k.none = (int)(cache_rows > 0 ? cache_rows : 1);
    k.scale_log2 = std::fmax(std::fabs(a->scale) * 1.4426950408889634f, 1e-30f);  // not 0: a masked score is -infinity times it
    k.negative = a->scale < 0;
    const bool bf = a->type == SIM_OP_BF16;
    CUtensorMap m, mq;
    const uint64_t size[2] = {(uint64_t)k.width, (uint64_t)k.none};
    const int64_t stride[1] = {a->blocks ? cache_row : k.width};
    const int64_t most_rows = (int64_t)a->new_tokens * a->heads;
    k.q_pad = most_rows <= 16 ? 16 : most_rows <= 32 ? 32 : kRows;
    const int col_blocks = (k.width + 63) / 64;
    auto stages_of = [&](int tile) { return (kShared - kRowBlockBytes - 1024 - col_blocks * k.q_pad * 128) / (col_blocks * tile * 128); };
    // Tiles of 64 tokens, whose scores take 1,208 cycles (of 32: 960).  Where only two
    // stages of 64 fit and one row tile leaves time to spare, five of 32 keep more
    // in flight: 3 x 90,001 to 130,000 tokens, rank 512 91.8 us, with 64 94.8.  Rank 384 68.7 us,
    // with 32 76.9; rank 256 59.2 (75.7); 64 requests of rank 512, 128 heads 105.5 (112).
    k.tile = c.row_tiles == 1 && stages_of(64) < 3 ? 32 : 64;
    k.stages = stages_of(k.tile);
    if (k.stages > kMostStages) k.stages = kMostStages;
    k.run = 4;
    while (k.run < k.tile && a->block_tokens % (2 * k.run) == 0) k.run *= 2;
    k.scattered = a->block_tokens % 4 != 0;
    const uint32_t box[2] = {64, k.scattered ? 1u : (uint32_t)k.run};
    if (!box_map(&m, a->blocks ? a->cache : a->q, bf, 2, size, stride, box)) return SIM_ERR_CUDA;
    // Q's (token, head) rows as one line
    const int64_t q_row = a->heads > 1 ? a->q_head : a->q_token;
    k.q_flat = a->new_tokens == 1 || a->heads == 1 || a->q_token == a->heads * a->q_head;
    {
        const uint64_t size[3] = {(uint64_t)k.width, (uint64_t)most_rows, (uint64_t)a->requests};
        const int64_t stride[2] = {most_rows > 1 && k.q_flat ? q_row : 8, a->requests > 1 ? a->q_request : 8};
        const uint32_t box[3] = {64, (uint32_t)k.q_pad, 1};
        if (!box_map(&mq, a->q, bf, 3, size, stride, box)) return SIM_ERR_CUDA;
    }
    const cudaStream_t st = (cudaStream_t)stream;
    return bf ? run<__nv_bfloat16>(k, m, mq, c, st) : run<__half>(k, m, mq, c, st);
}
