// What the operators' C entry points (kt_ops.cpp) and their kernels share.
#ifndef KT_OPS_INTERNAL_H
#define KT_OPS_INTERNAL_H

#include <stdint.h>

#include "kt_ops.h"

void kt_set_error(const char *fmt, ...);

constexpr int KT_ACT8_GROUP = 32;
constexpr int64_t kt_act8_groups(int64_t cols) { return (cols + KT_ACT8_GROUP - 1) / KT_ACT8_GROUP; }

// Launchers.  All return a hipError_t cast to int.
int kt_launch_layernorm_fwd(kt_dtype dt, kt_dtype pdt, int64_t rows, int cols, const void *x, int64_t ldx,
                            const void *gamma, const void *beta, float eps, void *y, int64_t ldy, float *mean,
                            float *rstd, int8_t *y8, uint8_t *e8, void *stream);
int64_t kt_layernorm_bwd_parts(int64_t rows, int64_t cols);
int kt_launch_layernorm_bwd(kt_dtype dt, kt_dtype pdt, int64_t rows, int cols, const void *dy, int64_t lddy,
                            const void *x, int64_t ldx, const int8_t *x8, const uint8_t *e8, const void *gamma,
                            const float *mean, const float *rstd, void *dx, int64_t lddx, void *dgamma, void *dbeta,
                            float *ws, void *stream);
int kt_launch_act8_save(kt_dtype dt, int64_t rows, int64_t cols, const void *x, int64_t ldx, int8_t *q, uint8_t *e,
                        void *stream);
int kt_launch_act8_restore(kt_dtype dt, int64_t rows, int64_t cols, const int8_t *q, const uint8_t *e, void *y,
                           int64_t ldy, void *stream);
int64_t kt_weight_grad_ws(kt_dtype dt, int64_t tokens, int64_t out, int64_t in);
int kt_launch_weight_grad(kt_dtype dt, kt_dtype gdt, int64_t tokens, int out, int in, const void *dy, int64_t lddy,
                          const int8_t *q, const uint8_t *e, void *dw, int64_t lddw, float *ws, void *stream);

// Lanes of attention's workgroups, and the queries or keys of one head that a workgroup owns.
constexpr int KT_ATTENTION_BLOCK = 256, KT_ATTENTION_OWN = 128;
int64_t kt_attention_bwd_ws(const kt_attention *a);
int kt_launch_attention_fwd(const kt_attention *a, const kt_heads *q, const kt_heads *k, const kt_heads *v, const kt_heads *o,
                            float *lse, void *stream);
int kt_launch_attention_bwd(const kt_attention *a, const kt_heads *d_o, const kt_heads *q, const kt_heads *k, const kt_heads *v,
                            const kt_heads *o, const float *lse, const kt_heads *dq, const kt_heads *dk, const kt_heads *dv,
                            float *ws, void *stream);

#endif
