/*
 * bdlm_norm.h -- C ABI of the normalisation between the attention layers (B200, sm_100a): layer norm or
 * root-mean-square norm of a residual stream, forward and backward.
 *
 * For T rows of D elements, with the residual's addition as part of the call:
 *     h = x + residual                 rounded to the element type; h = x without a residual
 *     mean = sum_d h_d / D             BDLM_NORM_LAYER (BDLM_NORM_RMS: 0)
 *     rstd = 1 / sqrt(sum_d (h_d - mean)^2 / D + eps)
 *     n = (h - mean) rstd,   y = n weight + bias
 * The statistics are those of h as it is stored, so that the backward, which reads h, is the derivative of what the
 * forward computed.  Backward, for the gradient dy of y and (optionally) the gradient dh that reaches h along the residual path:
 *     g = dy weight
 *     dx = rstd (g - mean_d(g) - n mean_d(g n)) + dh        (BDLM_NORM_RMS: without mean_d(g))
 *     dweight = sum_t dy n,   dbias = sum_t dy
 * dx is the gradient of x and of the residual alike.  All sums are held in fp32, every output is rounded once.
 *
 * Conventions as in bdlm_attn.h: device pointers, contiguous, owned by the caller, tensors 16-byte aligned (row statistics
 * 4-byte), work enqueued on `cuda_stream`, nothing allocated, 0 or a negative bdlm_status returned, arguments checked before
 * anything is launched.  T = 0 is a call without rows: dweight and dbias become zero, nothing else is written.
 *   x, residual, h, y, dy, dh, dx   [T, D]  of `dtype`
 *   weight, bias, dweight, dbias    [D]     of `wdtype` (the same as dtype, or BDLM_FP32)
 *   mean, rstd                      [T]     fp32
 * Outputs may overwrite inputs of the same shape and type element by element: y or h may be x or residual, dx may be dy or dh,
 * or h where a program no longer needs it.  Other overlaps are not allowed.
 */
#ifndef BDLM_NORM_H_
#define BDLM_NORM_H_

#include <stddef.h>
#include <stdint.h>

#include "bdlm_attn.h"
#include "bdlm_dtypes.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { BDLM_NORM_LAYER = 0, BDLM_NORM_RMS = 1 };
enum { BDLM_NORM_MAX_D = 32768 };

typedef struct {
  int32_t T, D;          /* 0 <= T <= 2^30, 1 <= D <= BDLM_NORM_MAX_D (BDLM_ERR_UNSUPPORTED above) */
  int32_t dtype;         /* BDLM_BF16, BDLM_FP16 or BDLM_FP32 */
  int32_t wdtype;        /* dtype or BDLM_FP32 */
  int32_t kind;          /* BDLM_NORM_LAYER or BDLM_NORM_RMS */
  float   eps;           /* >= 0; forward only */
  int32_t reserved[2];   /* 0 */
} bdlm_norm_params;

/* Scratch bytes of a backward that forms dweight (and dbias): fp32 partial sums of groups of rows, about one a multiprocessor.  0 where
 * none are needed (the smallest calls) and for invalid parameters. */
size_t bdlm_norm_workspace_bytes(const bdlm_norm_params* p);

/*
 * Forward.  weight NULL = 1, bias NULL = 0 (a bias needs a weight), residual NULL = none; h is written where there is a residual and has to be
 * given then (without one it must be NULL: it is x).  mean and rstd may be NULL where no backward follows; mean must be NULL
 * for BDLM_NORM_RMS.
 */
int bdlm_norm_fwd(const bdlm_norm_params* p, const void* x, const void* residual, const void* weight, const void* bias,
                  void* y, void* h, float* mean, float* rstd, void* cuda_stream);

/*
 * Backward.  weight as in the forward; mean must be given for BDLM_NORM_LAYER and NULL for BDLM_NORM_RMS.  dh NULL = 0.
 * dweight and dbias may be NULL (a weight that is not trained); with both NULL no workspace is needed.  The sums over the rows
 * run in a fixed order, so all gradients are bitwise reproducible; dx of a row does not depend on the other rows.
 */
int bdlm_norm_bwd(const bdlm_norm_params* p, const void* dy, const void* h, const void* weight, const float* mean,
                  const float* rstd, const void* dh, void* dx, void* dweight, void* dbias,
                  void* workspace, size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif  /* BDLM_NORM_H_ */
