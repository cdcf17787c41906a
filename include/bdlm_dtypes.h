/*
 * bdlm_dtypes.h -- element types of the operators that take more than one (bdlm_norm.h, bdlm_embed.h).
 */
#ifndef BDLM_DTYPES_H_
#define BDLM_DTYPES_H_

enum { BDLM_BF16 = 0, BDLM_FP16 = 1, BDLM_FP32 = 2 };

#endif  /* BDLM_DTYPES_H_ */
