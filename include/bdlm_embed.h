/*
 * bdlm_embed.h -- C ABI of the token embedding before the first layer (B200, sm_100a): rows of the table looked up and
 * scaled, and the table's gradient.
 *
 *     out_t = scale table[ids_t]                            rounded once
 *     dtable_v = scale sum_{t : ids_t = v} dout_t           (added to what dtable holds with accumulate = 1)
 * An id that is negative or not below V is no token (padding): its row of `out` is zero and it has no part in dtable.  The
 * gradient's sums are formed over the tokens sorted by id: in fp32, in an order that the ids alone fix, so they are
 * bitwise reproducible however often a token occurs (the mask token of block-diffusion training is half of all noisy
 * tokens).  A training step of block-diffusion looks up clean and noisy tokens of one table: as one call over both, or as a
 * second backward with accumulate = 1, which is also how the gradient of a table that is tied to the loss head is added to
 * the head's dW.
 *
 * Conventions as in bdlm_attn.h: device pointers, contiguous, owned by the caller, 16-byte aligned (ids 4-byte), work
 * enqueued on `cuda_stream`, nothing allocated, 0 or a negative bdlm_status returned, arguments checked before anything is launched.
 *   table, dtable   [V, D]  of `table_dtype`
 *   out, dout       [T, D]  of `out_dtype`: table_dtype, or any type where table_dtype is BDLM_FP32
 *   ids             [T]     int32
 * No output overlaps an input.  T = 0 is a call without tokens (dtable becomes zero, or stays as it is with accumulate = 1).
 */
#ifndef BDLM_EMBED_H_
#define BDLM_EMBED_H_

#include <stddef.h>
#include <stdint.h>

#include "bdlm_attn.h"
#include "bdlm_dtypes.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t T, D, V;       /* T >= 0; D, V >= 1; each at most 2^30 */
  int32_t table_dtype;   /* BDLM_BF16, BDLM_FP16 or BDLM_FP32 */
  int32_t out_dtype;
  float   scale;         /* finite */
  int32_t accumulate;    /* backward: 1 = add to dtable (rows of tokens that do not occur are not touched), 0 = overwrite all of it */
  int32_t reserved;      /* 0 */
} bdlm_embed_params;

/* Scratch bytes of the backward: the sorted tokens and fp32 sums of runs of equal tokens.  0 where none are needed (up to 32
 * tokens) and for invalid parameters. */
size_t bdlm_embed_workspace_bytes(const bdlm_embed_params* p);

int bdlm_embed_fwd(const bdlm_embed_params* p, const void* table, const int32_t* ids, void* out, void* cuda_stream);

int bdlm_embed_bwd(const bdlm_embed_params* p, const void* dout, const int32_t* ids, void* dtable,
                   void* workspace, size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif  /* BDLM_EMBED_H_ */
