// latent_prefill.cu -- causal attention of ragged requests with expanded keys
// and values (mtsim_ops.h).
#include "tensor.cuh"

#include <cmath>
#include <cooperative_groups.h>
#include <type_traits>
#include <cstddef>

namespace mtop {
namespace {

// One block computes 256 queries of one head of one request, as two tiles of
// 128 rows, over tiles of 128 keys:
//   S_t = Q_t K^T          (tensor core, 32-bit sums in tensor memory)
//   P_t = exp2(S_t - m)    (four warps a tile, one thread a row)
//   O_t += P_t V           (tensor core, P read from tensor memory)
// The tensor core alternates between the tiles, so that one tile's
// exponentials overlap the other's products.  K and V pass through a ring of
// 16 KB slots (128 rows of 64 elements) filled by bulk copies.  Bound by the
// tensor core and the thread that feeds it: a prompt of 8,192 tokens, 64 heads
// takes 865 to 905 us from GPU to GPU, 1.52 to 1.59 PFLOP/s.
constexpr int kRows = 128;              // of a tile of queries
constexpr int kQBytes = kRows * 128;    // of one column block (64 elements)
constexpr int kSlots = 8;
// TILES = 2: as above, with tiles of 128 keys.  TILES = 1: 128 queries over
// tiles of 64 keys, small enough for two blocks on a multiprocessor, so that
// one's start and end overlap the other's products: for short prompts.
template <int TILES> struct Shape {
    static constexpr int keys = 64 * TILES;
    static constexpr int slot_bytes = keys * 128;
    static constexpr int soft_warps = 4 * TILES;
    static constexpr int threads = (soft_warps + 4) * 32;  // + products, copies of K (and Q), zeros, copies of V
    static constexpr int q_slots = 3 * TILES;
    static constexpr int shared = q_slots * kQBytes + kSlots * slot_bytes + 256;
    // tensor memory columns: S (and P over its first half) and O of each tile
    static constexpr int col_s = 0, col_o = 128 * TILES, cols = 256 * TILES;
};
// Registers a thread with two tiles: 3 warpgroups launch with 168 (504 in all); the
// two of weights take 224, which holds a row's 128 scores without spilling.
constexpr int kSoftRegs = 224, kOtherRegs = 56;
constexpr uint32_t kHigh = operand_high(1024);

struct Args {
    const int32_t *q_offsets, *k_offsets;
    const void *value;
    void *out;
    float *lse;
    int64_t value_row, value_head, out_row, out_head;
    int q_rows, k_rows;
    int requests, heads, longest;
    int head_blocks, key_blocks, value_blocks;  // of 64 elements
    int value_dim;
    int causal;
    int groups;      // of heads that run side by side (their keys and values stay in L2)
    int row_blocks;  // of a block's queries
    int split;       // blocks that share queries
    float scale_log2, unscale;  // |scale| log2(e), and one over it
    bool negative;
};

// Few blocks and many keys: a cluster shares a block's queries, each of its
// blocks taking a stretch of the keys.  In the end each leaves its sums in
// shared memory, where Q and the first keys were, and joins a share of the rows.
constexpr int kMostSplit = 8;
constexpr int kSumsRow = SIM_OP_MAX_HEAD + 4;  // floats, so that eight rows lie in different banks
constexpr int kStatsOffset = 2 * kRows * kSumsRow * 4;
static_assert(kStatsOffset + 2 * kRows * 8 <= 6 * kQBytes + kSlots * Shape<2>::slot_bytes, "the sums fit where Q and the ring were");

constexpr int kInFlight = 4;  // tiles of K (and of V) in the ring: a tile of each takes 2 slots or more
struct Barriers {
    uint64_t q_full, k_full[kInFlight], k_empty[kInFlight], v_full[kInFlight], v_empty[kInFlight];
    uint64_t s_ready[2], p_ready[2], o_ready[2], v_cut, v_clean;  // v_cut: the last tile of V, if it has foreign rows
    uint32_t tmem;
    unsigned found;  // kNotFinite: a result is not finite; kLost: a wait has run out
};
static_assert(sizeof(Barriers) <= 256, "the room behind the ring");
constexpr unsigned kNotFinite = 1, kLost = 2;

// Sets up the barriers for a run over the keys (AGAIN: another one).
template <int TILES, bool AGAIN> __device__ __forceinline__ void init_barriers(Barriers *bars) {
    auto init = [](uint64_t *bar, uint32_t count) {
        if (AGAIN) bar_retire(smem_addr(bar));
        bar_init(smem_addr(bar), count);
    };
    init(&bars->q_full, 1);
    for (int s = 0; s < kInFlight; ++s) {
        init(&bars->k_full[s], 1), init(&bars->k_empty[s], 1);
        init(&bars->v_full[s], 1), init(&bars->v_empty[s], 1);
    }
    init(&bars->v_cut, 1), init(&bars->v_clean, 32);
    for (int t = 0; t < TILES; ++t) init(&bars->s_ready[t], 1), init(&bars->p_ready[t], kRows), init(&bars->o_ready[t], 1);
    bars->found = 0;
    bar_init_done();
}

template <typename T, int TILES, bool SPLIT>
__global__ void __launch_bounds__(Shape<TILES>::threads, 3 - TILES)
k_prefill(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap m_q, const __grid_constant__ CUtensorMap m_qr,
          const __grid_constant__ CUtensorMap m_k, const __grid_constant__ CUtensorMap m_kr,
          const __grid_constant__ CUtensorMap m_v) {
    using Z = Shape<TILES>;
    using R = WeightRange<T>;
    constexpr int kKeys = Z::keys, kSlotBytes = Z::slot_bytes, kSoftWarps = Z::soft_warps;
    constexpr int ring_offset = Z::q_slots * kQBytes;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t q_at = smem_addr(smem), ring = q_at + ring_offset;
    Barriers *bars = (Barriers *)(smem + ring_offset + kSlots * kSlotBytes);

    let_next_start();
    after_previous();
    // Which rows: a group of heads after another, in a group the last (longest)
    // row blocks of all requests first: 6 x 2,534 queries, 3 heads 40.8 us (a request
    // after another 49.8), 12 x 700, 8 heads 26.3 (31.9); short prompts with one tile take
    // either way the same.
    int item = SPLIT ? blockIdx.x / a.split : blockIdx.x;
    const int rank = SPLIT ? blockIdx.x % a.split : 0;
    int g0 = 0, in_group = a.heads;
    if (TILES == 2 && a.groups > 1) {
        const unsigned per_head = a.row_blocks * a.requests, g = (((unsigned)item / per_head + 1) * a.groups - 1) / a.heads;
        g0 = g * a.heads / a.groups, in_group = (g + 1) * a.heads / a.groups - g0;
        item -= g0 * per_head;
    }
    const int rest = item / in_group, h = g0 + item - rest * in_group, outer = rest / a.requests;
    const int b = rest - outer * a.requests, base = (a.row_blocks - 1 - outer) * TILES * kRows;
    const int q0 = min(max(a.q_offsets[b], 0), a.q_rows), q1 = min(a.q_offsets[b + 1], a.q_rows);
    int k0 = min(max(a.k_offsets[b], 0), a.k_rows);
    const int k1 = min(a.k_offsets[b + 1], a.k_rows);
    const int nq = q1 - q0, rows = min(nq, a.longest);
    int nk = max(k1 - k0, 0), behind = nk - nq;  // the first query sees `behind` + 1 keys
    if (base >= rows) return;
    const int start0 = base, start1 = base + kRows;
    auto tiles_for = [&](int start) {  // of keys, for the rows from `start` on
        if (start >= rows) return 0;
        const int sees = a.causal ? min(nk, min(start + kRows, rows) + behind) : nk;
        return sees > 0 ? (sees + kKeys - 1) / kKeys : 0;
    };
    int n0 = tiles_for(start0), n1 = TILES == 2 ? tiles_for(start1) : 0;
    if (SPLIT) {  // from here on, of this block's stretch of the keys
        const int share = (max(n0, n1) + a.split - 1) / a.split, first = rank * share;
        n0 = min(max(n0 - first, 0), share), n1 = min(max(n1 - first, 0), share);
        k0 += first * kKeys, nk -= first * kKeys, behind -= first * kKeys;
    }
    const int n = max(n0, n1);
    const int qk_blocks = a.head_blocks + a.key_blocks, per_tile = qk_blocks + a.value_blocks;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    bool dead = false;
    const bool cut = n > 0 && n * kKeys > nk;  // the last tile has rows that are not the request's
    // Keys that every row of the block sees, and the first tile with others.  A
    // row's weight of a key that it does not see is 0, but 0 times infinity or NaN is
    // not.  So where such tiles are and a result is not finite, the block does its
    // work again, this time with zeros in the place of infinities and NaN in these
    // tiles of V, and adds them to the rows that see them at the end.  The test
    // costs 0.7 to 4 % (8,192 tokens, 64 heads 877 us, 871 without; 37 prompts up to 300
    // 25.8, 24.9); zeros put there every time 2 to 12 %.
    const int all_see = max(a.causal ? min(nk, start0 + behind + 1) : nk, 0), open = min(n, all_see / kKeys);
    const bool may_redo = a.causal && open < n;
    bool redone = false;
    // All threads of the block, whose sums are out: whether the work is done again.
    auto redo = [&]() {
        if (dead) atomicOr(&bars->found, kLost);
        tmem_before_sync();
        asm volatile("bar.sync 1, %0;" ::"n"(Z::threads) : "memory");
        if (!may_redo || *(volatile unsigned *)&bars->found != kNotFinite) return false;
        asm volatile("bar.sync 1, %0;" ::"n"(Z::threads) : "memory");  // all have read it
        if (threadIdx.x == 0) init_barriers<TILES, true>(bars);
        asm volatile("bar.sync 1, %0;" ::"n"(Z::threads) : "memory");
        tmem_after_sync();
        return true;
    };

    if (threadIdx.x == 0) init_barriers<TILES, false>(bars);
    if (warp == kSoftWarps) tmem_alloc(smem_addr(&bars->tmem), Z::cols);
    if (threadIdx.x == (kSoftWarps + 1) * 32) fetch_map(&m_q), fetch_map(&m_qr), fetch_map(&m_k), fetch_map(&m_kr), fetch_map(&m_v);
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = bars->tmem;

    if (warp >= kSoftWarps) {
        if (TILES == 2) registers_down<kOtherRegs>();
        auto feed = [&]() {
            // ---------------------------------------------------------- copies
            // One warp for K (and Q), one for V, a lane a column block.  Eight slots
            // earlier in the stream lies a block of a fixed kind, a fixed number of tiles
            // back: when that has been used, the slot is free.
            if (warp == kSoftWarps + 1 && lane < Z::q_slots && n > 0) {
                const uint32_t qf = smem_addr(&bars->q_full);
                if (lane == 0) bar_expect(qf, ((n0 > 0) + (n1 > 0)) * qk_blocks * kQBytes);
                const int t = lane / 3, c = lane % 3, r = q0 + (t ? start1 : start0);
                const uint32_t dst = q_at + lane * kQBytes;
                if (c < qk_blocks && (t ? n1 : n0) > 0) {
                    if (c < a.head_blocks) copy_box_3d(dst, &m_q, 64 * c, h, r, qf);
                    else copy_box_3d(dst, &m_qr, 64 * (c - a.head_blocks), h, r, qf);
                }
            }
            if ((warp == kSoftWarps + 1 && lane < qk_blocks) || (warp == kSoftWarps + 3 && lane < a.value_blocks)) {
                const bool of_v = warp == kSoftWarps + 3;
                const int at = of_v ? qk_blocks + lane : lane;  // the block within a tile's blocks
                const int back = (kSlots - at + per_tile - 1) / per_tile;  // the slot's last block: of tile i - back
                const uint32_t empty = smem_addr(at - kSlots + back * per_tile < qk_blocks ? bars->k_empty : bars->v_empty);
                const uint32_t full = smem_addr(of_v ? bars->v_full : bars->k_full);
                const uint32_t bytes = (of_v ? a.value_blocks : qk_blocks) * kSlotBytes;
                const bool of_shared_key = !of_v && lane >= a.head_blocks;
                const CUtensorMap *map = of_v ? &m_v : of_shared_key ? &m_kr : &m_k;
                const int x = 64 * (of_shared_key ? lane - a.head_blocks : lane);
                int slot = at, r = k0;
                for (int i = 0; i < n; ++i, r += kKeys, slot = (slot + per_tile) % kSlots) {
                    const int old = i - back;
                    if (old >= 0) bar_wait(empty + old % kInFlight * 8, (old / kInFlight) & 1, dead);
                    const uint32_t bar = of_v && cut && i == n - 1 ? smem_addr(&bars->v_cut) : full + i % kInFlight * 8;
                    if (lane == 0) bar_expect(bar, bytes);
                    const uint32_t dst = ring + slot * kSlotBytes;
                    if (of_shared_key) copy_box_2d(dst, map, x, r, bar);
                    else copy_box_3d(dst, map, x, h, r, bar);
                }
            }
            if (warp == kSoftWarps + 2 && cut) {
                // rows of the last tile past the request's keys hold another's values: zeros, so that 0 * NaN cannot appear
                const int i = n - 1;
                bar_wait(smem_addr(&bars->v_cut), 0, dead);
                for (int c = 0; c < a.value_blocks; ++c) {
                    uint4 *rows_at = (uint4 *)(smem + ring_offset + (i * per_tile + qk_blocks + c) % kSlots * kSlotBytes + (nk - i * kKeys) * 128);
                    for (int e = lane; e < ((i + 1) * kKeys - nk) * 8; e += 32) rows_at[e] = make_uint4(0, 0, 0, 0);
                }
                fence_async();
                bar_arrive(smem_addr(&bars->v_clean));
            }
            // -------------------------------------------------------- products
            // One thread, and as few instructions as can be, each once: the tensor
            // core's queue is a product or two long, so what this thread executes (and
            // fetches) between two products is time in which the core stands still.
            if (warp == kSoftWarps && n > 0 && elect_one()) {
                const bool bf = std::is_same<T, __nv_bfloat16>::value;
                const uint32_t word_s = product_word(kRows, kKeys, bf, false, a.negative);
                const uint32_t word_o = product_word(kRows, 64 * a.value_blocks, bf, true, false);
                const uint32_t ring_k = operand_low(ring, 16), ring_v = operand_low(ring, kSlotBytes), q_0 = operand_low(q_at, 16);
                const uint32_t bar = smem_addr(bars);
                const uint32_t s_0 = tmem + Z::col_s, o_0 = tmem + Z::col_o;
                auto weighted = [&](int t, int slot, bool add) {  // O_t += P_t V, V's blocks from `slot` on
                    const uint32_t v = ring_v + slot * (kSlotBytes >> 4), p_at = s_0 + t * kRows, o_at = o_0 + t * kRows;
                    if (a.value_blocks == 2 && slot == kSlots - 1) {
                        // the two halves of V are not neighbours in the ring: one product each
                        const uint32_t word = product_word(kRows, 64, bf, true, false);
#pragma unroll 1
                        for (int e = 0; e < kKeys / 16; ++e) {
                            product_ts<kHigh>(o_at, p_at + 8 * e, v + 128 * e, word, add || e > 0);
                            product_ts<kHigh>(o_at + 64, p_at + 8 * e, ring_v + 128 * e, word, add || e > 0);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < kKeys / 16; ++e) product_ts<kHigh>(o_at, p_at + 8 * e, v + 128 * e, word_o, add || e > 0);
                    }
                };
                auto scores = [&](int t, int slot) {  // S_t = Q_t K^T, K's blocks from `slot` on
                    uint32_t q = q_0 + t * (3 * kQBytes >> 4);
#pragma unroll 1
                    for (int c = 0; c < qk_blocks; ++c, q += kQBytes >> 4) {
                        const uint32_t k = ring_k + ((slot + c) & 7) * (kSlotBytes >> 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) product_ss<kHigh, kHigh>(s_0 + t * kRows, q + 2 * e, k + 2 * e, word_s, c + e > 0);
                    }
                    product_commit(bar + offsetof(Barriers, s_ready) + t * 8);
                };
                auto wait_k = [&](int i) { bar_wait(bar + offsetof(Barriers, k_full) + (i & 3) * 8, (i >> 2) & 1, dead); };
                auto wait_v = [&](int i) {
                    if (cut && i == n - 1) bar_wait(bar + offsetof(Barriers, v_clean), 0, dead);
                    else bar_wait(bar + offsetof(Barriers, v_full) + (i & 3) * 8, (i >> 2) & 1, dead);
                };
                auto wait_p = [&](int t, int i) {
                    bar_wait(bar + offsetof(Barriers, p_ready) + t * 8, i & 1, dead);
                    tmem_after_sync();
                };
                auto free_k = [&](int i) { product_commit(bar + offsetof(Barriers, k_empty) + (i & 3) * 8); };
                auto free_v = [&](int i) { product_commit(bar + offsetof(Barriers, v_empty) + (i & 3) * 8); };

                bar_wait(bar + offsetof(Barriers, q_full), 0, dead);
                wait_k(0);
                if (n0 > 0) scores(0, 0);
                if (n1 > 0) scores(1, 0);
                wait_v(0);
                int v_slot = qk_blocks & 7, k_slot = per_tile & 7;  // of V of tile i, of K of tile i + 1
                int i = 0;
                // While both tiles go on.  What is not urgent (slots given back, the wait
                // for the next V) comes where the core has products queued.
                for (; TILES == 2 && i + 1 < min(n0, n1); ++i) {
                    wait_p(0, i);
                    weighted(0, v_slot, i > 0);
                    free_k(i);
                    wait_k(i + 1);
                    scores(0, k_slot);
                    wait_p(1, i);
                    weighted(1, v_slot, i > 0);
                    free_v(i);
                    wait_v(i + 1);
                    scores(1, k_slot);
                    v_slot = (v_slot + per_tile) & 7, k_slot = (k_slot + per_tile) & 7;
                }
                // Tiles that only some rows see.
#pragma unroll 1
                for (; i < n; ++i) {
                    free_k(i);
                    if (i + 1 < n) wait_k(i + 1);
#pragma unroll 1
                    for (int t = 0; t < TILES; ++t) {
                        const int nt = t ? n1 : n0;
                        if (i >= nt) continue;
                        wait_p(t, i);
                        weighted(t, v_slot, i > 0);
                        if (i + 1 == nt) product_commit(bar + offsetof(Barriers, o_ready) + t * 8);
                        else scores(t, k_slot);
                    }
                    free_v(i);
                    if (i + 1 < n) wait_v(i + 1);
                    v_slot = (v_slot + per_tile) & 7, k_slot = (k_slot + per_tile) & 7;
                }
                bar_wait(bar + offsetof(Barriers, v_empty) + ((n - 1) & 3) * 8, ((n - 1) >> 2) & 1, dead);  // every arrival has come
            }
            __syncwarp();
        };
        feed();
        redone = redo();
        if (redone) feed();
        if (SPLIT) {
            cluster_sync();
            cluster_sync();
        }
    } else {
        if (TILES == 2) registers_up<kSoftRegs>();
        // ------------------------------------------------- weights and sums
        const int t = warp / 4, row = (t ? start1 : start0) + (warp % 4) * 32 + lane;
        const int nt = t ? n1 : n0;
        const int sees = a.causal ? min(nk, row + behind + 1) : nk;  // keys [0, sees) of this row
        const int first_sees = a.causal ? min(nk, row - lane + behind + 1) : nk;  // of the warp's first row: the fewest
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t s_at = tmem + Z::col_s + t * kRows + lanes, o_at = tmem + Z::col_o + t * kRows + lanes;
        const float scale = a.scale_log2;
        // A tile's infinities and NaN that not every row sees become zeros.  (With two
        // tiles of queries the other four warps do the same, and leave the same bytes.)
        auto clean = [&](int i) {
            if (cut && i == n - 1) bar_wait(smem_addr(&bars->v_cut), 0, dead);
            else bar_wait(smem_addr(&bars->v_full[i % kInFlight]), (i / kInFlight) & 1, dead);
            const int first = max(all_see - i * kKeys, 0) * 8, own = min(nk - i * kKeys, kKeys) * 8;  // in 16 bytes
#pragma unroll 1
            for (int c = 0; c < a.value_blocks; ++c) {
                uint4 *at = (uint4 *)(smem + ring_offset + (i * per_tile + qk_blocks + c) % kSlots * kSlotBytes);
#pragma unroll 1
                for (int e = first + threadIdx.x % kRows; e < own; e += kRows) {
                    const uint4 w = at[e], f = make_uint4(finite_only<T>(w.x), finite_only<T>(w.y), finite_only<T>(w.z), finite_only<T>(w.w));
                    if (w.x != f.x || w.y != f.y || w.z != f.z || w.w != f.w) at[e] = f;
                }
            }
            fence_async();
            __syncwarp();
        };
        // What the row sees of them is added to its sums.
        auto add_cleaned = [&]() {
            const T *value = (const T *)a.value + (int64_t)k0 * a.value_row + h * a.value_head;
#pragma unroll 1
            for (int c = 0; 32 * c < a.value_dim; ++c) {
                uint32_t o[32];
                tmem_ld32(o_at + 32 * c, o);
                tmem_wait_ld();
#pragma unroll 1
                for (int j = all_see; j < min(sees, nt * kKeys); ++j) {
                    const T *v = value + j * a.value_row + 32 * c;
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float x = 32 * c + e < a.value_dim ? elem<T>::to(v[e]) : 0.f;
                        if (!(fabsf(x) < INFINITY)) o[e] = __float_as_uint(__uint_as_float(o[e]) + x);
                    }
                }
                __syncwarp();
                tmem_st32(o_at + 32 * c, o);
            }
            tmem_wait_st();
        };
        auto weights = [&](auto second) {
            constexpr bool again = decltype(second)::value;
            float top = -INFINITY, sum = 0.f;  // top: of the scaled scores, as far as P has been scaled by it
            for (int i = 0; i < nt; ++i) {
                if (again && i >= open) clean(i);
                bar_wait(smem_addr(&bars->s_ready[t]), (uint32_t)i & 1, dead);
                tmem_after_sync();
                uint32_t s[kKeys];
#pragma unroll
                for (int c = 0; c < kKeys / 32; ++c) tmem_ld32(s_at + 32 * c, s + 32 * c);
                tmem_wait_ld();
                float *x = (float *)s;
                if ((i + 1) * kKeys > first_sees) {
                    const int v = sees - i * kKeys;
#pragma unroll
                    for (int c = 0; c < kKeys; ++c)
                        if (c >= v) x[c] = -INFINITY;
                }
                float m0 = x[0], m1 = x[1], m2 = x[2], m3 = x[3];
#pragma unroll
                for (int c = 4; c < kKeys; c += 4) {
                    m0 = fmaxf(m0, x[c]), m1 = fmaxf(m1, x[c + 1]), m2 = fmaxf(m2, x[c + 2]), m3 = fmaxf(m3, x[c + 3]);
                }
                const float high = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * scale;
                // The sums are rescaled only when the maximum has grown by 2^grow:
                // until then weights up to that are as exact, and O stays where it is.
                const bool grow = high > top + R::grow;
                if (__any_sync(~0u, grow || beyond_fused(top))) {
                    const float keep = grow ? exp2_fast(top - high) : 1.f;
                    if (grow) top = high;
                    sum *= keep;
                    if (beyond_fused(top)) {
#pragma unroll
                        for (int c = 0; c < kKeys; ++c) x[c] = below_top(x[c], scale, top) * a.unscale;  // times the scale again below
                    }
                    if (i > 0) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (32 * c < 64 * a.value_blocks) {
                                uint32_t o[32];
                                tmem_ld32(o_at + 32 * c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                                tmem_st32(o_at + 32 * c, o);
                            }
                        }
                    }
                }
                const float base = beyond_fused(top) ? R::raise : R::raise - top;
                float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
                uint32_t p[kKeys / 2];
#pragma unroll
                for (int c = 0; c < kKeys; c += 4) {
                    float e0, e1, e2, e3;
                    fma2(e0, e1, x[c], x[c + 1], scale, scale, base, base);
                    fma2(e2, e3, x[c + 2], x[c + 3], scale, scale, base, base);
                    e0 = exp2_fast(e0), e1 = exp2_fast(e1), e2 = exp2_fast(e2), e3 = exp2_fast(e3);
                    add2(s0, s1, e0, e1);
                    add2(s2, s3, e2, e3);
                    p[c / 2] = pack2<T>(e0, e1);
                    p[c / 2 + 1] = pack2<T>(e2, e3);
                }
                tmem_st32(s_at, p);
                if (TILES == 2) tmem_st32(s_at + 32, p + kKeys / 2 - 32);
                tmem_wait_st();
                tmem_before_sync();
                bar_arrive(smem_addr(&bars->p_ready[t]));
                sum += (s0 + s1) + (s2 + s3);
            }
            uint32_t bad = 0, bad2 = 0;
            if (nt > 0) {
                bar_wait(smem_addr(&bars->o_ready[t]), 0, dead);
                tmem_after_sync();
                if (again && nt > open) add_cleaned();
            }
            if (SPLIT) {
                // every product has read what the sums overwrite
                if (n0 > 0) bar_wait(smem_addr(&bars->o_ready[0]), 0, dead);
                if (n1 > 0) bar_wait(smem_addr(&bars->o_ready[1]), 0, dead);
                tmem_after_sync();
                const int local = t * kRows + (warp % 4) * 32 + lane;
                ((float2 *)(smem + kStatsOffset))[local] = make_float2(top, sum);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (32 * c < 64 * a.value_blocks && nt > 0) {
                        uint32_t o[32];
                        tmem_ld32(o_at + 32 * c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *(uint4 *)(smem + ((size_t)local * kSumsRow + 32 * c + e) * 4) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                        if (sum != 0.f && row < rows)
#pragma unroll
                            for (int e = 0; e < 32; ++e) bad |= !(fabsf(__uint_as_float(o[e])) < INFINITY);
                    }
                }
                fence_async();  // (bulk copies write there when the work is done again)
            } else {
                // a sum of 0 is a row that sees nothing: zeros; a sum that is no number stays one
                if (row < rows && a.lse)
                    a.lse[(int64_t)(q0 + row) * a.heads + h] = sum != 0.f ? (top + (log2f(sum) - R::raise)) * 0.6931471805599453f : -INFINITY;
                const float inv = sum != 0.f ? 1.f / sum : 0.f;
                T *out = (T *)a.out + (int64_t)(q0 + row) * a.out_row + h * a.out_head;
#pragma unroll 1
                for (int c = 0; c < 2 * a.value_blocks; ++c) {
                    uint32_t o[32];
                    if (nt > 0) {
                        tmem_ld32(o_at + 32 * c, o);
                        tmem_wait_ld();
                    }
                    if (row < rows) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            if (32 * c + e < a.value_dim) {
                                uint4 w;
                                auto val = [&](int j) { return sum != 0.f ? __uint_as_float(o[e + j]) * inv : 0.f; };
                                w.x = pack2<T>(val(0), val(1)), w.y = pack2<T>(val(2), val(3));
                                w.z = pack2<T>(val(4), val(5)), w.w = pack2<T>(val(6), val(7));
                                *(uint4 *)(out + 32 * c + e) = w;
                                spoil<T>(bad, w.x), spoil<T>(bad2, w.y), spoil<T>(bad, w.z), spoil<T>(bad2, w.w);
                            }
                    }
                }
            }
            if (!again && spoiled(bad | bad2) && may_redo) atomicOr(&bars->found, kNotFinite);
            __syncwarp();
        };
        weights(std::false_type());
        redone = redo();
        if (redone) weights(std::true_type());
        if (SPLIT) {
            cluster_sync();
            // A warp takes four rows at a time: lane 8 j + k has the factor of block
            // k's sums of row j, then each lane four elements of all four rows.
            const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
            const int there = min(TILES * kRows, rows - base), k8 = lane % kMostSplit;
            for (int r0 = rank + a.split * 4 * warp; r0 < there; r0 += a.split * 4 * kSoftWarps) {
                const int mine = r0 + a.split * (lane / kMostSplit);
                float2 st = make_float2(-INFINITY, 0.f);
                if (k8 < a.split && mine < there) st = ((const float2 *)cluster.map_shared_rank(smem + kStatsOffset, k8))[mine];
                float top = st.x;
#pragma unroll
                for (int o = kMostSplit / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
                // sums of 0 count as nothing (they may not have been written)
                const float f = st.y == 0.f ? 0.f : exp2_fast(st.x - (top == -INFINITY ? 0.f : top));
                const unsigned some = __ballot_sync(~0u, st.y != 0.f);
                float sum = st.y == 0.f ? 0.f : f * st.y;
#pragma unroll
                for (int o = kMostSplit / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                float4 v[4] = {};
#pragma unroll 2
                for (int k = 0; k < a.split; ++k) {
                    const char *at = (const char *)cluster.map_shared_rank(smem, k) + (r0 * kSumsRow + 4 * lane) * 4;
                    float4 u[4] = {};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (some >> (kMostSplit * j + k) & 1) u[j] = *(const float4 *)(at + j * a.split * kSumsRow * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float w = __shfl_sync(~0u, f, kMostSplit * j + k);
                        v[j].x = fmaf(w, u[j].x, v[j].x), v[j].y = fmaf(w, u[j].y, v[j].y);
                        v[j].z = fmaf(w, u[j].z, v[j].z), v[j].w = fmaf(w, u[j].w, v[j].w);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float all = __shfl_sync(~0u, sum, kMostSplit * j), inv = all != 0.f ? 1.f / all : 0.f;
                    const int r = r0 + j * a.split;
                    if (r < there && 4 * lane < a.value_dim)
                        *(uint2 *)((T *)a.out + (int64_t)(q0 + base + r) * a.out_row + h * a.out_head + 4 * lane) =
                            make_uint2(pack2<T>(v[j].x * inv, v[j].y * inv), pack2<T>(v[j].z * inv, v[j].w * inv));
                }
                if (a.lse && k8 == 0 && mine < there)
                    a.lse[(int64_t)(q0 + base + mine) * a.heads + h] = sum != 0.f ? (top + (log2f(sum) - R::raise)) * 0.6931471805599453f : -INFINITY;
            }
            __syncwarp();
            cluster_sync();  // the others have read
        }
    }
    if (redone) {
        __syncwarp();
        tmem_before_sync();
        __syncthreads();
    }
    if (warp == kSoftWarps) tmem_free(tmem, Z::cols);
}

template <typename T, int TILES, bool SPLIT>
int run(const Args &k, const CUtensorMap *m, unsigned grid, cudaStream_t st) {
    static std::atomic<uint64_t> told;
    if (!allow_shared((const void *)k_prefill<T, TILES, SPLIT>, Shape<TILES>::shared, told)) return SIM_ERR_CUDA;
    const cudaError_t e = launch_early(k_prefill<T, TILES, SPLIT>, grid, Shape<TILES>::threads, Shape<TILES>::shared, k.split, st, k, m[0], m[1], m[2], m[3], m[4]);
    return launched("sim_op_latent_prefill", e);
}

}  // namespace

unsigned prefill_faults() {
    unsigned n = 0;
    return cudaMemcpyFromSymbol(&n, g_faults, sizeof n) == cudaSuccess ? n : ~0u;
}

}  // namespace mtop

using namespace mtop;

extern "C" int sim_op_latent_prefill(const sim_op_latent_prefill_t *a, void *stream) {
    if (!a) return fail(SIM_ERR_ARG, "args is NULL");
    if (a->type != SIM_OP_BF16 && a->type != SIM_OP_FP16) return fail(SIM_ERR_ARG, "element type %d: 16-bit types only", a->type);
    if (a->requests < 0 || a->heads < 0 || a->longest < 0 || a->q_rows < 0 || a->k_rows < 0)
        return fail(SIM_ERR_ARG, "sizes must not be negative");
    if (a->head_dim < 8 || a->head_dim > SIM_OP_MAX_HEAD || a->head_dim % 8)
        return fail(SIM_ERR_ARG, "head_dim must be a multiple of 8 in [8, %d]", SIM_OP_MAX_HEAD);
    if (a->key_dim < 0 || a->key_dim > SIM_OP_MAX_KEY || a->key_dim % 8)
        return fail(SIM_ERR_ARG, "key_dim must be a multiple of 8 in [0, %d]", SIM_OP_MAX_KEY);
    if (a->value_dim < 8 || a->value_dim > SIM_OP_MAX_HEAD || a->value_dim % 8)
        return fail(SIM_ERR_ARG, "value_dim must be a multiple of 8 in [8, %d]", SIM_OP_MAX_HEAD);
    if (a->causal != 0 && a->causal != 1) return fail(SIM_ERR_ARG, "causal must be 0 or 1");
    if (!std::isfinite(a->scale)) return fail(SIM_ERR_ARG, "scale must be finite");
    if (a->requests == 0 || a->longest == 0 || a->heads == 0 || a->q_rows == 0) return SIM_OK;
    if (a->q_rows > INT32_MAX - 65536 || a->k_rows > INT32_MAX - 65536 || a->heads > 65535 || a->requests > 65535)
        return fail(SIM_ERR_ARG, "rows must be below 2^31 - 2^16, heads and requests at most 65535");
    if (!a->q || !a->out || !a->q_offsets || !a->k_offsets || (a->k_rows && (!a->key || !a->value || (a->key_dim && !a->shared))))
        return fail(SIM_ERR_ARG, "q, key, shared, value, the offsets and out must not be NULL");
    const int64_t heads = a->heads;
    if (!aligned16(a->q) || !aligned16(a->key) || (a->key_dim && (!aligned16(a->shared) || !even_stride(a->k_rows, a->shared_row))) ||
        !aligned16(a->value) || !aligned16(a->out) || !even_stride(a->q_rows, a->q_row) || !even_stride(heads, a->q_head) ||
        !even_stride(a->k_rows, a->key_row) || !even_stride(heads, a->key_head) || !even_stride(a->k_rows, a->value_row) ||
        !even_stride(heads, a->value_head) || !even_stride(a->q_rows, a->out_row) || !even_stride(heads, a->out_head))
        return fail(SIM_ERR_ARG, "tensors must be aligned to 16 bytes, with strides that are multiples of 8 elements");
    const bool bf = a->type == SIM_OP_BF16;
    Args k;
    k.q_offsets = a->q_offsets, k.k_offsets = a->k_offsets, k.value = a->value, k.out = a->out, k.lse = a->lse;
    k.value_row = a->value_row, k.value_head = a->value_head;
    k.out_row = a->out_row, k.out_head = a->out_head, k.q_rows = (int)a->q_rows, k.k_rows = (int)a->k_rows;
    k.requests = a->requests, k.heads = a->heads, k.longest = a->longest;
    k.head_blocks = (a->head_dim + 63) / 64, k.key_blocks = (a->key_dim + 63) / 64, k.value_blocks = (a->value_dim + 63) / 64;
    k.value_dim = a->value_dim, k.causal = a->causal;
    k.scale_log2 = std::fmax(std::fabs(a->scale) * 1.4426950408889634f, 1e-30f);  // not 0: a masked score is -infinity times it
    k.unscale = 1.f / k.scale_log2;
    k.negative = a->scale < 0;
    const int64_t longest = a->longest < a->q_rows ? a->longest : a->q_rows;
    // One tile a block where most prompts leave the second one empty and keys
    // are few: 37 ragged prompts up to 300, 16 heads 24.8 us (two tiles 32.7), 64 x 128
    // tokens, 64 heads 133 us (197); two tiles for the rest: 37 x 512 tokens 102 us (one
    // 122), 16 x 256 tokens after up to 1,000 cached ones 77.5 us (96).
    const int tiles = longest <= 384 && a->q_rows <= 192 * (int64_t)a->requests && a->k_rows <= 384 * (int64_t)a->requests ? 1 : 2;
    k.row_blocks = (int)((longest + tiles * kRows - 1) / (tiles * kRows));
    // Heads side by side: as many as keep their keys and values within about a third of L2.
    const int64_t head_bytes = a->k_rows * (a->head_dim + a->value_dim) * 2;
    const int64_t fit = head_bytes > 0 ? (40 << 20) / head_bytes : a->heads;
    k.groups = (int)(fit < 1 ? a->heads : (a->heads + fit - 1) / fit);  // of equal size, or one apart: a last group of few heads would leave a long tail
    // Keys are split where blocks would leave half of the SMs empty, by as much as
    // keeps all blocks resident (of clusters of 8 there is room for fewer than 16).
    // 16 heads of 1,000 queries after 2,728 cached tokens: 51.7 us, two stretches 36.3
    // (four 46.5); 16 heads of 200 after 1,033: 22.2, two 20.1, four 16.8 (eight 29.2); 4 x
    // 2,048: 30.1, four 19.1; 4 heads of 200 after 1,100: 22.7, four 15.7, eight 15.4.  The
    // join takes 3 to 5 us, most where two blocks do it: 16 x 1,024 queries alone 19.1, two 19.3;
    // 16 heads of 200 after 216: 13.0, four 13.1; after 97: 11.5, four 12.7.
    const int sms = sm_count();
    if (!sms) return SIM_ERR_CUDA;
    k.split = 1;
    if (tiles == 2) {
        const int64_t some = a->q_rows / (2 * kRows) + a->requests, most = (int64_t)a->requests * k.row_blocks;
        const int64_t blocks = (some < most ? some : most) * a->heads;
        k.split = blocks * 8 <= sms / 2 ? 8 : blocks * 4 <= sms ? 4 : blocks * 2 <= sms ? 2 : 1;
        if (a->k_rows < (int64_t)a->requests * (k.split == 2 ? 1280 : 448)) k.split = 1;
    }
    const int64_t grid = (int64_t)a->requests * k.row_blocks * a->heads * k.split;
    if (grid > INT32_MAX) return fail(SIM_ERR_ARG, "requests * heads * longest is too large");

    CUtensorMap m[5];
    const int keys = 64 * tiles;
    auto map3 = [&](CUtensorMap *to, const void *base, int dim, int64_t rows, int64_t head, int64_t row, int box_rows) {
        const uint64_t size[3] = {(uint64_t)dim, (uint64_t)a->heads, (uint64_t)(rows > 0 ? rows : 1)};
        const int64_t stride[2] = {a->heads > 1 ? head : 8, rows > 1 ? row : 8};
        const uint32_t box[3] = {64, 1, (uint32_t)box_rows};
        return box_map(to, base, bf, 3, size, stride, box);
    };
    const char *q_key = (const char *)a->q + 2 * a->head_dim;
    bool ok = map3(&m[0], a->q, a->head_dim, a->q_rows, a->q_head, a->q_row, kRows) &&
              map3(&m[1], a->key_dim ? q_key : a->q, a->key_dim ? a->key_dim : 8, a->q_rows, a->q_head, a->q_row, kRows);
    // without keys nothing is copied: any valid map does
    const void *key = a->k_rows ? a->key : a->q, *value = a->k_rows ? a->value : a->q;
    ok = ok && map3(&m[2], key, a->head_dim, a->k_rows, a->key_head, a->key_row, keys) &&
         map3(&m[4], value, a->value_dim, a->k_rows, a->value_head, a->value_row, keys);
    if (ok) {
        const bool has = a->k_rows && a->key_dim;
        const uint64_t size[2] = {has ? (uint64_t)a->key_dim : 8u, has ? (uint64_t)a->k_rows : 1u};
        const int64_t stride[1] = {has && a->k_rows > 1 ? a->shared_row : 8};
        const uint32_t box[2] = {64, (uint32_t)keys};
        ok = box_map(&m[3], has ? a->shared : a->q, bf, 2, size, stride, box);
    }
    if (!ok) return SIM_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    const unsigned g = (unsigned)grid;
    if (tiles == 1) return bf ? run<__nv_bfloat16, 1, false>(k, m, g, st) : run<__half, 1, false>(k, m, g, st);
    if (k.split > 1) return bf ? run<__nv_bfloat16, 2, true>(k, m, g, st) : run<__half, 2, true>(k, m, g, st);
    return bf ? run<__nv_bfloat16, 2, false>(k, m, g, st) : run<__half, 2, false>(k, m, g, st);
}
