/*
 * tcu_lm.h - C ABI of the language-model operators of the tensor-core-unit library (B200, sm_100a).
 *
 * Beside the plain scans of tcu_scan.h:
 *
 *  - Linear attention with a constant decay for each head: an inclusive scan whose elements are dk x dv matrices.
 *    Per sequence and head, with a = exp(log_decay[head]) and a state S of dk x dv values,
 *        S_t = a S_{t-1} + k_t v_t^T            o_t = scale * S_t^T q_t
 *    in chunks: the scan inside a chunk is a product with a triangular matrix of powers of a, the carry between
 *    chunks is the state.  Prompts (with states in and out, dense or packed), training (gradients), single tokens.
 *  - Token embedding: out[n] = scale * table[ids[n]], and its table gradient, a segmented sum over the tokens in
 *    the order of their ids.
 *
 * The general conventions of tcu_scan.h hold: caller-owned device memory, nothing allocated, everything asynchronous
 * on `stream`, argument errors found on the host before anything is queued, bounded device-side waits, launches that
 * can be captured into a CUDA graph.
 */
#ifndef TCU_LM_H_
#define TCU_LM_H_

#include "tcu_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types of tokens, tables and gradients */
typedef enum { TCU_F32 = 0, TCU_F16 = 1, TCU_BF16 = 2 } tcu_float_t;

/* A (batch, token, head, feature) array: features are contiguous, the other strides are given in elements.  Any order of
 * batch, token and head is a choice of strides; a stride of 0 repeats an input along that axis (not along tokens).
 * In the packed form (d_offsets given) stride_batch is not used. */
typedef struct {
    void *ptr;
    int64_t stride_batch, stride_token, stride_head;
} tcu_tokens_t;

/* Arguments of the linear-attention calls.  Zero-initialise, set struct_bytes = sizeof(tcu_linattn_t), then set what
 * the call uses.  States are fp32, (batch, heads, dk, dv) dense. */
typedef struct {
    uint32_t struct_bytes;
    uint32_t type;              /* TCU_F16 or TCU_BF16: q, k, v, o and their gradients                              */
    uint64_t batch;             /* sequences                                                                        */
    uint64_t tokens;            /* tokens of each sequence; packed: of all sequences together; step: not used       */
    uint32_t heads, dk, dv;     /* dk, dv: 1 to 128                                                                 */
    float scale;                /* a factor on every output                                                         */
    const float *d_log_decay;   /* `heads` values, log of the decay of each head (-inf: no memory; values above 0 let
                                   the state grow and are the caller's concern; NaN: outputs, states and gradients
                                   of the head are NaN, other heads are not affected)                              */
    const int64_t *d_offsets;   /* NULL: dense.  Packed: batch + 1 values, sequence b holds tokens [offsets[b],
                                   offsets[b+1]); non-decreasing, first 0, last `tokens` (not checked: they live on the device); empty
                                   sequences are allowed                                                            */
    const int32_t *d_slots;     /* step only: NULL, or for each sequence its entry in the state pool; entries below
                                   0 or at or above pool_slots mark a sequence to skip (its output is zero, no state
                                   is touched); no two sequences may share an entry                                 */
    uint64_t pool_slots;        /* step only: entries of the pool (at least `batch` when d_slots is NULL)           */
    tcu_tokens_t q, k, v, o;    /* o: written by forward and step                                                   */
    const float *d_state_in;    /* NULL (zero), or the state before the first token                                 */
    float *d_state_out;         /* NULL, or receives the state after the last token (may be d_state_in itself, but
                                   not overlap it otherwise); step: the pool, updated in place                      */
    tcu_tokens_t d_o;           /* backward: gradient with respect to o                                             */
    tcu_tokens_t d_q, d_k, d_v; /* backward: receive the gradients (per head, also where an input has a stride of 0:
                                   sum over the repeated axis afterwards); no element of one may be an element of
                                   another (looked at only where they begin at the same address)                    */
    const float *d_dstate_out;  /* backward: NULL (zero), or the gradient with respect to the state after the last token */
    float *d_dstate_in;         /* backward: NULL, or receives the gradient with respect to the state before the first */
    void *d_scratch;            /* forward and backward: NULL, or tcu_linattn_scratch_bytes() of 256-byte aligned memory, with
                                   which many heads, or packed sequences of different lengths, are
                                   spread evenly over the SMs; needs no clearing; not to be shared by
                                   calls that may overlap                                                           */
    uint64_t scratch_bytes;     /* size of it                                                                       */
} tcu_linattn_t;

/* Workspace of the forward and backward calls: the status of bounded waits (tcu_scan_device_status reads it).  Clear it
 * once with tcu_scan_workspace_init; any number of calls, concurrent ones too, may share it.  It may lie in page-locked host memory
 * as well, where the host clears it (zeros), and reads without waiting what its third 32-bit word holds: 0, or TCU_ERR_TIMEOUT. */
size_t tcu_linattn_workspace_bytes(void);

/* Bytes of scratch with which a forward (or backward) call with these arguments runs faster; 0 if it would not, as when there are
 * no more sequences times heads (backward: three times that) than SMs.  Looks at sizes alone (whether d_offsets is given among them). */
size_t tcu_linattn_scratch_bytes(const tcu_linattn_t *args, int backward);

/* o and, if asked for, the state after the last token.
 *   q, k, v, o  16-byte aligned pointers, strides multiples of 8 elements; the bytes from o's first element to its last must not overlap an input's
 *   batch 0, or 0 tokens: nothing but states is written
 * TCU_ERR_UNSUPPORTED: dk or dv above 128, more than 2^31 - 256 tokens, more than 2^31 - 1 blocks of work.
 * Non-finite values: a product with a non-finite k or v reaches every output of its sequence that shares the token's group of
 * 128 tokens (counted from the start of the sequence), earlier ones too; other sequences never see it.  Tokens past the
 * end of a packed sequence are never part of it, whatever they hold.
 * float16: scores, keys and states are brought to the type's range inside, so that only inputs and outputs are bound by it; states
 * up to 2^75, and keys times scale from 2^-55 on, keep their 32 bits. */
tcu_status_t tcu_linattn_forward(const tcu_linattn_t *args, void *d_ws, size_t ws_bytes, cudaStream_t stream);

/* Gradients with respect to q, k, v and the state before the first token, from d_o and d_dstate_out.  Reads q, k, v, d_o, d_state_in;
 * o and d_state_out are not used.  With D_t the gradient with respect to S_t:
 *     D_t = scale * q_t do_t^T + a D_{t+1},  dq_t = scale * S_t do_t,  dk_t = D_t v_t,  dv_t = D_t^T k_t
 * The decays are constants of the model: no gradient with respect to them is computed. */
tcu_status_t tcu_linattn_backward(const tcu_linattn_t *args, void *d_ws, size_t ws_bytes, cudaStream_t stream);

/* Self-test of the ways in which these calls give up (compare tcu_scan_selftest_timeout): the ordinary forward (or backward) call,
 * except that group `silent_group` (128 tokens each, counted from 0 as the block that walks them comes to them) of every walk never
 * reports its part of the state as done, and that every device-side wait gives up after `limit_ms` milliseconds (1..1000)
 * instead of about a second.  The kernel winds down and returns; after the stream has drained, tcu_scan_device_status(d_ws) is
 * TCU_ERR_TIMEOUT if any walk has so many groups, outputs and states are not valid, and tcu_scan_workspace_init clears the condition. */
tcu_status_t tcu_linattn_selftest_timeout(const tcu_linattn_t *args, int backward, uint32_t silent_group, unsigned limit_ms, void *d_ws,
                                          size_t ws_bytes, cudaStream_t stream);

/* One token for each of `batch` sequences: the state of each (an entry of the pool d_state_out, (pool_slots, heads, dk, dv)) is
 * updated in place, and o written.  q, k, v, o: stride_token is not used; any alignment of elements.  The pool: 16-byte
 * aligned.  Needs no workspace.  o may be v, with its strides; its elements must not be elements of q or k (which is looked at only
 * where they begin at the same address), nor of another head's or sequence's v: blocks read and write in any order. */
tcu_status_t tcu_linattn_step(const tcu_linattn_t *args, cudaStream_t stream);

/* out[n][0..d) = scale * table[ids[n]][0..d): products in fp32, rounded once to the type.
 *   d_ids      device, n values of 4 or 8 bytes (id_bytes), signed; an id outside [0, rows) gives a row of zeros
 *   d_table    device, rows x d, row stride table_stride elements (at most 2^38);  d_out  device, n x d dense, of the same type */
tcu_status_t tcu_embedding_forward(const void *d_ids, int id_bytes, size_t n, const void *d_table, size_t rows, size_t d,
                                   size_t table_stride, tcu_float_t type, float scale, void *d_out, cudaStream_t stream);

/* d_table[v] = scale * (sum of d_out[n] over the n with ids[n] = v), for every row v: rows that no token names are set to
 * zero, or, with accumulate = 1, the sums are added to what the table holds and no other row is touched.
 * The tokens are sorted by id (stable), the rows of a run are added in fp32 in the order of the tokens in blocks whose bounds
 * depend on the ids alone: the result is the same from call to call, bit by bit.
 *   d_out       device, n x d dense, of `type`;  d_ids as above, ids outside [0, rows) are left out
 *   d_table     device, rows x d dense, of `table_type`: fp32, or the same as `type`
 *   d_ws        tcu_embedding_workspace_bytes(n, rows, d) bytes, 256-byte aligned; needs no clearing; not to be shared
 *               by calls that may overlap
 * TCU_ERR_UNSUPPORTED: n or rows above 2^30 - 1, d above 2^20, a table_type other than fp32 and `type`. */
size_t tcu_embedding_workspace_bytes(size_t n, size_t rows, size_t d);
tcu_status_t tcu_embedding_backward(const void *d_out, tcu_float_t type, const void *d_ids, int id_bytes, size_t n, size_t rows,
                                    size_t d, float scale, int accumulate, void *d_table, tcu_float_t table_type,
                                    void *d_ws, size_t ws_bytes, cudaStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* TCU_LM_H_ */
