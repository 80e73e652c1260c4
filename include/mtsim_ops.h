/*
 * mtsim_ops.h -- C ABI of the operators of one instance's iteration, in
 * libmtsim beside the simulation (mtsim.h).
 *
 * The simulation charges an iteration base + a * prefill tokens + b * decode
 * requests microseconds.  The paper's simulator takes such times from operator
 * run times profiled on a GPU (Sec. 2.5, 4.1); these entry points are the
 * operators to profile: what an instance does in an iteration with its
 * block-paged cache (T tokens per block) when every cached token is one
 * latent vector shared by all heads, followed by one rotated key part.
 *
 *   sim_op_rotary          rotary positions on part of every head
 *   sim_op_latent_append   a token's latent vector and rotated key into the cache
 *   sim_op_latent_decode   attention of new tokens over the cache (absorbed form)
 *   sim_op_latent_prefill  causal attention with expanded keys and values
 *   sim_op_sample          temperature, top-k, top-p, min-p and the draw
 *
 * Conventions for every entry point:
 *  - The argument struct is host memory and may be reused when the call
 *    returns; every pointer inside it is device memory of the current device,
 *    owned by the caller, and must stay valid until the work is done.
 *  - Work is queued on cuda_stream (a cudaStream_t, NULL = legacy default
 *    stream).  No call synchronises, allocates or keeps anything, so each may be
 *    captured into a graph after one call of its kind on the device.
 *  - Return value: SIM_OK (0), SIM_ERR_ARG or SIM_ERR_CUDA (mtsim.h);
 *    sim_op_last_error() then describes the failure.  Nothing is queued when
 *    SIM_ERR_ARG is returned.
 *  - Strides are in elements.  A tensor's last dimension is contiguous.  The
 *    stride of a dimension of one element is not used; inputs may have strides of 0.
 *  - Values on the device (lengths, tables, slots, offsets) cannot be checked
 *    on the host: each kernel bounds them as stated, so that no value reaches
 *    memory outside the tensors.
 *  - Results do not depend on the stream, on other work or on the run: the
 *    same inputs give the same bits.
 */
#ifndef MTSIM_OPS_H
#define MTSIM_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "mtsim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define SIM_OP_BF16 0
#define SIM_OP_FP16 1
#define SIM_OP_FP32 2

/* Layout of the pairs in a rotated part of d elements: pair i is elements
 * (2i, 2i+1), or (i, i + d/2). */
#define SIM_OP_INTERLEAVED 0
#define SIM_OP_HALF 1

#define SIM_OP_MAX_ROT 256      /* elements of a head's rotated part */
#define SIM_OP_MAX_RANK 512     /* elements of a latent vector */
#define SIM_OP_MAX_KEY 64       /* elements of the shared rotated key of attention */
#define SIM_OP_MAX_HEAD 128     /* elements of a head's own key part, and of its values */
#define SIM_OP_MAX_VOCAB (1 << 20)

/* Rotary positions.  With d = rot_dim, o = rot_offset, p = positions[n] and
 * the pairs (a, b) of x[n][h][o .. o+d):
 *   a' = amplitude * (a cos(p f_i) - b sin(p f_i))
 *   b' = amplitude * (a sin(p f_i) + b cos(p f_i))
 * inverse = 1 turns the other way (the gradient's rotation, or a key's
 * position taken out again).  The other elements of the head are copied.
 * frequencies[i] (d/2 of them, 64-bit) are radians per position; scalings for
 * long contexts are scalings of them and of amplitude.  The angle is reduced
 * exactly (in 2^-64 turns), so it is as good at position 2^31 - 1 as at 1. */
typedef struct {
    const void *x;              /* [tokens][heads][dim] */
    void *out;                  /* same shape and type; may be x itself with x's strides */
    const void *positions;      /* [tokens], 32- or 64-bit signed */
    const double *frequencies;  /* [rot_dim / 2] */
    int64_t tokens;
    int64_t x_token, x_head;    /* strides of x */
    int64_t out_token, out_head;
    int32_t heads, dim;
    int32_t rot_dim, rot_offset; /* even, at most SIM_OP_MAX_ROT; rot_offset + rot_dim <= dim */
    int32_t type, layout;
    int32_t positions_64;       /* 1: 64-bit positions */
    int32_t inverse;
    float amplitude;
} sim_op_rotary_t;

int sim_op_rotary(const sim_op_rotary_t *args, void *cuda_stream);

/* Writes rows of the block cache: row slots[n] (block slots[n] / T, row
 * slots[n] % T) becomes [latent[n], rotated key[n]], the key rotated as above
 * with amplitude.  A slot outside [0, blocks * T) writes nothing (padding).
 * Two tokens of one call must not name the same slot. */
typedef struct {
    const void *latent;         /* [tokens][rank] */
    const void *key;            /* [tokens][rot_dim] */
    void *cache;                /* [blocks][block_tokens][rank + rot_dim] */
    const void *positions;      /* [tokens], 32- or 64-bit signed */
    const int64_t *slots;       /* [tokens] */
    const double *frequencies;  /* [rot_dim / 2] */
    int64_t tokens;
    int64_t latent_token, key_token; /* strides */
    int64_t cache_block, cache_row;
    int64_t blocks;
    int32_t block_tokens;       /* T >= 1 */
    int32_t rank, rot_dim;      /* rank >= 1, any; rot_dim even, at most SIM_OP_MAX_ROT */
    int32_t type, layout;
    int32_t positions_64;
    float amplitude;
} sim_op_latent_append_t;

int sim_op_latent_append(const sim_op_latent_append_t *args, void *cuda_stream);

/* Attention of each request's last `new_tokens` tokens over its cached
 * tokens, queries already taken into the latent space (absorbed form).  With
 * W = rank + key_dim, cached row j of request b being c_j (row j % T of block
 * table[b][j / T]) and L = lengths[b] (the new tokens included):
 *   s_j = scale * <q[b][t][h], c_j>   for j < L - new_tokens + 1 + t
 *   lse[b][t][h] = log sum_j exp s_j
 *   out[b][t][h] = sum_j exp(s_j - lse) c_j[0 .. rank)
 * A row that sees nothing, or only scores of -infinity, gives zeros and lse = -infinity; one whose scores
 * are NaN or +infinity gives NaN.  lengths are taken
 * as at most table_blocks * T; a table entry outside [0, blocks) stands for a
 * block of zeros.  Cached rows from L on are never used, whatever they hold,
 * and a new token's result has no part of those after it.
 * Scores, statistics and sums are in 32 bits; only the weights exp(s - max)
 * are rounded to the inputs' type, for their product with c (a tensor-core
 * operand; their sum is of the unrounded ones, so lse keeps 32 bits): each by at
 * most 2^-9 (bfloat16) or 2^-12 (float16) of itself, a float16 one below 2^-24
 * by at most 2^-35.  Types: 16-bit.  Alignment: pointers and strides of q and cache are multiples of 16 bytes (8 elements), rank a multiple of 64, key_dim of 8;
 * cache_block is a multiple of cache_row (a cache that is one layer of several is).
 * workspace: sim_op_latent_decode_workspace() bytes for the same sizes,
 * 256-byte aligned, contents need not be set; not to be shared by calls that overlap. */
typedef struct {
    const void *q;              /* [requests][new_tokens][heads][rank + key_dim] */
    const void *cache;          /* [blocks][block_tokens][rank + key_dim] */
    const int32_t *table;       /* [requests][table_blocks], rows `table_row` apart */
    const int32_t *lengths;     /* [requests] */
    void *out;                  /* [requests][new_tokens][heads][rank] */
    float *lse;                 /* [requests][new_tokens][heads], contiguous, or NULL */
    void *workspace;
    size_t workspace_bytes;
    int64_t q_request, q_token, q_head; /* strides */
    int64_t out_request, out_token, out_head;
    int64_t cache_block, cache_row, table_row;
    int64_t blocks;
    int32_t requests, new_tokens, heads;
    int32_t rank, key_dim;
    int32_t block_tokens, table_blocks;
    int32_t type;
    float scale;
} sim_op_latent_decode_t;

int sim_op_latent_decode(const sim_op_latent_decode_t *args, void *cuda_stream);
size_t sim_op_latent_decode_workspace(int32_t requests, int32_t new_tokens, int32_t heads, int32_t rank);

/* Causal attention of ragged requests with expanded keys and values: request
 * b has queries [q_offsets[b], q_offsets[b+1]) and keys [k_offsets[b],
 * k_offsets[b+1]), Q and K of them; query i sees key j when j <= i + K - Q
 * (its own token is the last it sees; the K - Q keys before are its cached
 * prefix), or every key with causal = 0.  Scores are
 *   s_ij = scale * (<q[i][h][0 .. head_dim), key[j][h]> + <q[i][h][head_dim ..), shared[j]>)
 * with the rotated key `shared` common to all heads; out and lse as above.
 * Keys and values that a query does not see have no part in its result, whatever
 * they hold (a call with infinities or NaN in tokens that some queries see and
 * others not takes up to twice the time).
 * Offsets must not decrease; they are bounded by q_rows and k_rows, and at
 * most `longest` queries of a request are computed (`longest` also decides,
 * with the numbers of rows, requests and heads, how the work is cut, and so the last bits).  Rows that belong to no
 * request are not written.  Types: 16-bit.  Alignment: pointers and strides of
 * q, key, shared, value and out are multiples of 16 bytes; head_dim, key_dim
 * and value_dim are multiples of 8. */
typedef struct {
    const void *q;              /* [q_rows][heads][head_dim + key_dim] */
    const void *key;            /* [k_rows][heads][head_dim] */
    const void *shared;         /* [k_rows][key_dim] */
    const void *value;          /* [k_rows][heads][value_dim] */
    const int32_t *q_offsets;   /* [requests + 1] */
    const int32_t *k_offsets;   /* [requests + 1] */
    void *out;                  /* [q_rows][heads][value_dim] */
    float *lse;                 /* [q_rows][heads], contiguous, or NULL */
    int64_t q_row, q_head;      /* strides */
    int64_t key_row, key_head, shared_row, value_row, value_head;
    int64_t out_row, out_head;
    int64_t q_rows, k_rows;
    int32_t requests, heads, longest;
    int32_t head_dim, key_dim, value_dim; /* at most SIM_OP_MAX_HEAD, SIM_OP_MAX_KEY, SIM_OP_MAX_HEAD */
    int32_t causal;
    int32_t type;
    float scale;
} sim_op_latent_prefill_t;

int sim_op_latent_prefill(const sim_op_latent_prefill_t *args, void *cuda_stream);

/* One token per row of logits.  With t the row's temperature, m its largest
 * logit and w_i = exp((l_i - m) / t), held in units of 2^-40:
 *   1. top_k > 0 keeps the top_k largest logits;
 *   2. top_p < 1 then keeps, from the largest down, each token before which
 *      less than top_p of the kept weight lies (so always the first);
 *   3. min_p > 0 keeps the tokens with w_i >= min_p (above 1: as 1);
 *   4. the token is the first, in vocabulary order, up to which the kept
 *      weights sum to more than uniform times their total.
 * Equal logits rank by index, the lowest first.  A temperature that is not
 * above zero takes the largest logit (the lowest index of them) whatever the
 * rest says.  NaN logits count as -infinity.  With infinite logits the weight
 * is shared by the +infinite ones.  A row without a logit above -infinity
 * gives token -1 and log-probability -infinity.  logprob is the logarithm of
 * the drawn token's share of the kept weight.  Parameter arrays may be NULL
 * (temperature 1, no limits). */
typedef struct {
    const void *logits;         /* [rows][vocab] */
    const float *uniform;       /* [rows], in [0, 1) */
    const float *temperature;   /* [rows] or NULL */
    const int32_t *top_k;       /* [rows] or NULL; <= 0 and >= vocab: no limit */
    const float *top_p;         /* [rows] or NULL; >= 1: no limit */
    const float *min_p;         /* [rows] or NULL */
    int64_t *token;             /* [rows] */
    float *logprob;             /* [rows] or NULL */
    int64_t logits_row;         /* stride */
    int32_t rows, vocab;        /* vocab in [1, SIM_OP_MAX_VOCAB] */
    int32_t type;
} sim_op_sample_t;

int sim_op_sample(const sim_op_sample_t *args, void *cuda_stream);

/* Number of waits inside the operators' kernels that ran out of their limit
 * on the current device since the library was loaded: 0, unless a kernel is
 * at fault (its results are then not to be used).  Synchronises the device.
 * Negative: SIM_ERR_CUDA. */
int sim_op_faults(void);

/* Text of the last error of an operator on this thread. */
const char *sim_op_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* MTSIM_OPS_H */
