/*
 * pvconv_train.h -- C ABI of the operators around the networks' point MLPs
 * that training and 8-bit serving use: group normalisation with an activation,
 * linear layers in 8-bit floating point and in 8-bit integers, the distillation
 * loss against a teacher's top logits, and the cross entropy of a linear layer,
 * each with its gradients.
 *
 * The conventions of pvconv.h hold for every call here: device pointers owned
 * by the caller, rows of channels with a row stride in elements (`*_ld`, 0
 * means "= number of channels"), arguments checked on the host before anything
 * is enqueued, the same status codes, no allocation, no synchronisation, no
 * state between calls. Workspaces are 256-byte aligned and hold nothing
 * between calls. Outputs may not overlap inputs. Results are the same bits on
 * every run (no floating-point atomics). A call can be captured in a HIP graph.
 */
#ifndef PVCONV_TRAIN_H
#define PVCONV_TRAIN_H

#include "pvconv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PVCONV_MAX_NORM_CHANNELS 16384
#define PVCONV_FP8_BLOCK 128          /* values that share one scale */
#define PVCONV_FP8_MAX_CHANNELS 65536
#define PVCONV_MAX_TOP 256            /* teacher entries a row */
#define PVCONV_MAX_CLASSES (1 << 24)

/* ------------------------------------------------------------------------- */
/* Group normalisation and an activation, channels last.                     */
/*                                                                           */
/* Over cloud b's first n rows (n = lengths[b], or N) and the C / groups     */
/* channels of a group: mean, var = mean of (x - mean)^2, and                */
/*   y = act( gamma_c * (x - mean) / sqrt(var + eps) + beta_c ).             */
/* Rows from n on are not read as values and y is 0 there (n = 0: the whole  */
/* cloud; a length outside [0, N] is clamped). The statistics are summed in  */
/* 64 bits, about a value of the group or its mean, and kept in 32.          */
/*  x        [B][N][C] (x_dt), row k of cloud b at (b*N + k) * x_ld          */
/*  lengths  [B] int32 or NULL                                               */
/*  gamma, beta  [C] fp32                                                    */
/*  act      NONE, RELU, LEAKY (slope) or SILU                               */
/*  y        out [B][N][C] (y_dt), row stride y_ld                           */
/*  stats    out [B][groups][2] fp32: mean, 1 / sqrt(var + eps) (0, 0 for an */
/*           empty cloud), or NULL                                           */
/* groups divides C; 1 <= C <= PVCONV_MAX_NORM_CHANNELS; B*N <= 2^30.        */
/* ------------------------------------------------------------------------- */
size_t pvconv_group_norm_act_workspace_size(int B, int N, int C, int groups);
pvconv_status pvconv_group_norm_act(const void* x, pvconv_dtype x_dt, int x_ld, int B, int N,
                                    int C, int groups, const int32_t* lengths,
                                    const float* gamma, const float* beta, float eps,
                                    pvconv_act act, float slope, void* y, pvconv_dtype y_dt,
                                    int y_ld, float* stats, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* Its gradients, from x and the statistics of the forward. With             */
/* xh = (x - mean) * rstd, v = gamma xh + beta, dv = dy * act'(v) (act' of   */
/* the rectifiers read from the sign of v: 1 where v > 0, else slope or 0):  */
/*   dgamma_c = sum dv xh,  dbeta_c = sum dv  over every valid row,          */
/*   dx = rstd (gamma dv - mean_g(gamma dv) - xh mean_g(gamma dv xh)),       */
/* 0 in rows past a cloud's length. The sums are 32-bit over a workgroup's   */
/* share of a cloud's rows and 64-bit over the shares.                       */
/*  dy  [B][N][C] (dy_dt), row stride dy_ld;  dx out (dx_dt), dx_ld          */
/*  dgamma, dbeta  out [C] fp32, or NULL                                     */
size_t pvconv_group_norm_act_backward_workspace_size(int B, int N, int C, int groups);
pvconv_status pvconv_group_norm_act_backward(
    const void* dy, pvconv_dtype dy_dt, int dy_ld, const void* x, pvconv_dtype x_dt, int x_ld,
    int B, int N, int C, int groups, const int32_t* lengths, const float* stats,
    const float* gamma, const float* beta, pvconv_act act, float slope, void* dx,
    pvconv_dtype dx_dt, int dx_ld, float* dgamma, float* dbeta, void* workspace,
    size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- */
/* Linear layer in 8-bit floating point (OCP e4m3), a scale for each block   */
/* of 128 values.                                                            */
/*                                                                           */
/* A block is quantised as q = e4m3(v * 2^-e), to nearest, ties to even, with */
/* e the smallest whole number >= -126 such that the block's largest finite  */
/* |v| <= 448 * 2^e (e = 0 for a block of zeros); its scale is the byte      */
/* e + 127. A value that is not finite becomes NaN and does not count for    */
/* the largest. Power-of-two scales lose no digits and are what the scaled   */
/* matrix instructions of gfx950 take.                                       */
/*                                                                           */
/* Sums. An fp32 output (dw always is one) has fp32 sums of exact products,  */
/* but that a quantised value below 2^-133 is rounded to a multiple of it.   */
/* For a bf16 output the matrix instruction adds the 128 products of a block */
/* on a grid that the largest of them sets, and the blocks in fp32: within   */
/* 2^-12 of the sum of the products' magnitudes (5e-5 measured), where e4m3  */
/* itself has rounded each factor by up to 2^-4. Where that matters (sums    */
/* that cancel), ask for an fp32 output.                                     */
/*                                                                           */
/* Layouts (K128 = K rounded up to a multiple of 128, padding is zero):      */
/*   weight     [N][K128] bytes, scale [N128/128][K128/128]: blocks 128 x 128 */
/*   weight_t   [K][N128] bytes, scale_t [K128/128][N128/128]: the transpose, */
/*              the same blocks and scales                                   */
/* ------------------------------------------------------------------------- */

/* w [N][K] (w_dt), row stride w_ld -> weight, scale, and weight_t, scale_t  */
/* unless those two are NULL. 16-byte aligned byte arrays.                    */
pvconv_status pvconv_fp8_quantize_weight(const void* w, pvconv_dtype w_dt, int w_ld, int N,
                                         int K, uint8_t* weight, uint8_t* scale,
                                         uint8_t* weight_t, uint8_t* scale_t, void* stream);

/* y[m,n] = act( sum_k Q(x)[m,k] W[n,k] + bias_n ), Q in blocks of 128        */
/* consecutive channels of a row.                                            */
/*  x     [M][K] (x_dt), row stride x_ld                                     */
/*  bias  [N] fp32 or NULL; act NONE, RELU or LEAKY (slope)                  */
/*  y     out [M][N] (y_dt), row stride y_ld                                 */
/* 1 <= K, N <= PVCONV_FP8_MAX_CHANNELS; M/128 * max(K, N)/128 (rounded up)  */
/* <= 2^26. weight 16-byte aligned.                                          */
size_t pvconv_fp8_linear_workspace_size(int M, int K, int N);
pvconv_status pvconv_fp8_linear(const void* x, pvconv_dtype x_dt, int x_ld, int M, int K, int N,
                                const uint8_t* weight, const uint8_t* scale, const float* bias,
                                pvconv_act act, float slope, void* y, pvconv_dtype y_dt,
                                int y_ld, void* workspace, size_t workspace_bytes,
                                void* stream);

/* The gradients of y = x W^T + bias:                                        */
/*   dx = Q(dy) W          Q: blocks of 128 consecutive channels of a row    */
/*   dw = Qc(dy)^T Qc(x)   Qc: blocks of 128 consecutive rows of a channel   */
/*   dbias_n = sum_m dy[m,n]  (not quantised)                                */
/*  dy [M][N] (dy_dt), dy_ld; x [M][K] (x_dt), x_ld                          */
/*  dx out [M][K] (dx_dt), dx_ld, or NULL (weight_t, scale_t then unused)    */
/*  dw out [N][K] fp32 or NULL (x then unused); dbias out [N] fp32 or NULL   */
size_t pvconv_fp8_linear_backward_workspace_size(int M, int K, int N);
pvconv_status pvconv_fp8_linear_backward(const void* dy, pvconv_dtype dy_dt, int dy_ld,
                                         const void* x, pvconv_dtype x_dt, int x_ld, int M,
                                         int K, int N, const uint8_t* weight_t,
                                         const uint8_t* scale_t, void* dx, pvconv_dtype dx_dt,
                                         int dx_ld, float* dw, float* dbias, void* workspace,
                                         size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- */
/* Linear layer in 8-bit integers, a scale for each row of x and for each row */
/* (output channel) of the weight.                                           */
/*                                                                           */
/* A row v is quantised with the scale s, the smallest bf16 number >= 2^-126 */
/* with 127 s >= its largest |v|: q = the whole number nearest to v / s, ties */
/* to even (in real arithmetic: any implementation gives these bytes). A row */
/* that holds a NaN or an infinity has the scale NaN and q = 0.              */
/* Eight bits of a scale cost at most 2^-7 of the range and make products of */
/* scales, and of a scale and a bf16 value, exact.                           */
/*                                                                           */
/* Layout: q [R][K128] bytes, scale [R] fp32 (K128 = K rounded up to a       */
/* multiple of PVCONV_INT8_BLOCK; padding is written as zero and has to be). */
/* Byte arrays are 16-byte aligned.                                          */
/* ------------------------------------------------------------------------- */
#define PVCONV_INT8_BLOCK 128         /* quantised rows are whole blocks */
#define PVCONV_INT8_MAX_CHANNELS 65536

/* x [R][K] (x_dt), row stride x_ld -> q, scale: of a weight [N][K], of rows. */
/* 0 <= R <= 2^30, 1 <= K <= PVCONV_INT8_MAX_CHANNELS.                       */
pvconv_status pvconv_int8_quantize(const void* x, pvconv_dtype x_dt, int x_ld, int R, int K,
                                   int8_t* q, float* scale, void* stream);

/* y[m,n] = act( s_m scale_n sum_k q[m,k] weight[n,k] + bias_n ), q and s of x's */
/* rows. The sums are exact integers, rounded once to fp32.                  */
/*  x     [M][K] (x_dt), row stride x_ld                                     */
/*  bias  [N] fp32 or NULL; act NONE, RELU or LEAKY (slope)                  */
/*  y     out [M][N] (y_dt), row stride y_ld                                 */
/*  rows, row_scale  out: x's quantised rows, kept for the backward and for  */
/*        pvconv_int8_linear_rows in x's place, or NULL (both). A call that  */
/*        keeps them takes pvconv_int8_linear_rows_workspace_size.           */
/* 1 <= K, N <= PVCONV_INT8_MAX_CHANNELS; M/128 * max(K, N)/128 (rounded up) */
/* <= 2^26.                                                                  */
size_t pvconv_int8_linear_workspace_size(int M, int K, int N);
pvconv_status pvconv_int8_linear(const void* x, pvconv_dtype x_dt, int x_ld, int M, int K, int N,
                                 const int8_t* weight, const float* scale, const float* bias,
                                 pvconv_act act, float slope, void* y, pvconv_dtype y_dt,
                                 int y_ld, int8_t* rows, float* row_scale, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* The same layer of rows that are quantised already: the bits of the call that */
/* quantised them.                                                           */
size_t pvconv_int8_linear_rows_workspace_size(int M, int K, int N);
pvconv_status pvconv_int8_linear_rows(const int8_t* rows, const float* row_scale, int M, int K,
                                      int N, const int8_t* weight, const float* scale,
                                      const float* bias, pvconv_act act, float slope, void* y,
                                      pvconv_dtype y_dt, int y_ld, void* workspace,
                                      size_t workspace_bytes, void* stream);

/* The gradients of y = x W^T + bias at the quantised values x = s q, W =    */
/* scale weight, from the kept rows:                                         */
/*   dx[m,k] = sum_n dy[m,n] scale_n weight[n,k]                             */
/*   dw[n,k] = sum_m dy[m,n] row_scale_m rows[m,k],  dbias_n = sum_m dy[m,n] */
/* Sums are fp32, of products that are exact (bf16 dy) or good to 24 bits    */
/* (fp32 dy; for a bf16 dx, dy scale_n is rounded to 16 bits first). scale_n  */
/* weight and dy row_scale are formed in 32 bits and should be finite there.  */
/*  dy [M][N] (dy_dt), dy_ld; dx out [M][K] (dx_dt), dx_ld, or NULL (weight, */
/*  scale then unused); dw out [N][K] fp32 or NULL (rows, row_scale then     */
/*  unused); dbias out [N] fp32 or NULL                                      */
size_t pvconv_int8_linear_backward_workspace_size(int M, int K, int N);
pvconv_status pvconv_int8_linear_backward(const void* dy, pvconv_dtype dy_dt, int dy_ld,
                                          const int8_t* rows, const float* row_scale, int M,
                                          int K, int N, const int8_t* weight,
                                          const float* scale, void* dx, pvconv_dtype dx_dt,
                                          int dx_ld, float* dw, float* dbias, void* workspace,
                                          size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- */
/* Distillation from a teacher's top logits.                                 */
/*                                                                           */
/* Row m has student logits z [V], a teacher's `top` entries (value t_j,     */
/* class i_j; an entry whose class is outside [0, V) is absent) and a label. */
/* With p = softmax(t / T) over the present entries, q = softmax(z / T):     */
/*   loss_m = alpha T^2 sum_j p_j (log p_j - log q_{i_j})                    */
/*            + (1 - alpha) (logsumexp(z) - z_label),                        */
/* the first term 0 for a row without teacher entries (none present, or all  */
/* present values -inf), the second for a label outside [0, V) or labels     */
/* NULL; both 0, and no gradient, for a row whose logits are all -inf. An    */
/* entry with p_j = 0 adds nothing; entries of one class add up. A NaN or    */
/* +inf logit makes the terms of its row NaN. Where alpha > 0, z / T is      */
/* taken in 32 bits: at T < 1 a logit may be infinite over T, and counts as  */
/* that.                                                                     */
/*  z        [M][V] (z_dt), row stride z_ld                                  */
/*  t_val    [M][top] fp32, t_class [M][top] int32, contiguous               */
/*  labels   [M] int32 or NULL;  temperature > 0, it and its inverse finite  */
/*           in 32 bits;  0 <= alpha <= 1                                    */
/*  loss     out [M] fp32                                                    */
/*  lse      out [M][2] fp32 or NULL: logsumexp(z), logsumexp(z / T), 0 in   */
/*           the place of one whose term has no weight (labels NULL or       */
/*           alpha = 1; alpha = 0)                                           */
/*           Loss and gradient are of these 32-bit values and carry their    */
/*           rounding: q of a row whose maximum is of size 2^k is good to    */
/*           2^(k-24). Rows masked whole by a type's lowest value have no    */
/*           digit left; mask them by -inf, or give them the weight 0.       */
/*  dz       out [M][V] (dz_dt), row stride dz_ld, or NULL: row_weight[m]    */
/*           (1 if NULL) times d loss_m / d z. A row of weight 0 is 0.       */
/* 1 <= V <= PVCONV_MAX_CLASSES, 1 <= top <= PVCONV_MAX_TOP, M <= 2^30.      */
/* The workspace size is 0 and the workspace is not looked at: sums stay in  */
/* registers and LDS.                                                        */
/* ------------------------------------------------------------------------- */
size_t pvconv_distill_topk_workspace_size(int M, int V);
pvconv_status pvconv_distill_topk(const void* z, pvconv_dtype z_dt, int z_ld, int M, int V,
                                  const float* t_val, const int32_t* t_class, int top,
                                  const int32_t* labels, float temperature, float alpha,
                                  const float* row_weight, float* loss, float* lse, void* dz,
                                  pvconv_dtype dz_dt, int dz_ld, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* The gradient alone, from the lse of a forward with the same arguments;    */
/* dloss [M] fp32 (or NULL: 1) in the place of row_weight.                   */
pvconv_status pvconv_distill_topk_backward(const void* z, pvconv_dtype z_dt, int z_ld, int M,
                                           int V, const float* t_val, const int32_t* t_class,
                                           int top, const int32_t* labels, float temperature,
                                           float alpha, const float* lse, const float* dloss,
                                           void* dz, pvconv_dtype dz_dt, int dz_ld,
                                           void* stream);

/* ------------------------------------------------------------------------- */
/* Softmax cross entropy of a linear layer's outputs, without the logits.    */
/*                                                                           */
/* With z = x W^T + bias (never in memory whole: a piece of the classes at a  */
/* time), a row m of label l:                                                */
/*   lse_m = logsumexp(z_m),  loss_m = lse_m - z_ml,                         */
/*   dz_m = row_weight_m (softmax(z_m) - onehot(l)),                         */
/*   dx = dz W,  dw = dz^T x,  dbias_v = sum_m dz[m,v].                      */
/* A label outside [0, V): loss and dz are 0. So they are for a row whose    */
/* logits are all -inf; a class whose logit is -inf (by its bias) takes no   */
/* part. A NaN or +inf logit makes its row's lse, loss and dz NaN. A row of  */
/* weight 0 has dz = 0; x and W should be finite all the same, as dz         */
/* multiplies them.                                                          */
/* fp32 operands are multiplied to 24 bits, bf16 ones exactly, sums are fp32, */
/* an exponential is off by 2^-24 |z - lse| of itself. What of a factor of a  */
/* gradient lies below 2^-133 is left out: row weights below some 2^-110 cost */
/* digits.                                                                   */
/* For a bf16 dx (dw), dz and an fp32 W (x) are rounded to 16 bits first; for */
/* an fp32 one they are taken to 24.                                         */
/*  x       [M][K] (x_dt), row stride x_ld;  w [V][K] (w_dt), row stride w_ld */
/*  bias    [V] fp32 or NULL;  labels [M] int32;  row_weight [M] fp32 or     */
/*          NULL (1)                                                         */
/*  loss    out [M] fp32;  lse out [M] fp32 or NULL, for the backward        */
/*  dx      out [M][K] (dx_dt), dx_ld;  dw out [V][K] (dw_dt), contiguous;   */
/*          dbias out [V] fp32; each NULL where not wanted                   */
/* 0 <= M <= 2^24, 1 <= K <= PVCONV_CE_MAX_CHANNELS, 1 <= V <=               */
/* PVCONV_MAX_CLASSES. The workspace sizes are those of a call with every    */
/* gradient (want_grad) or none; for a backward, want_grad. They hold x and W */
/* in parts (2 bytes a bf16 value, 6 an fp32 one, K up to 64s; not used for   */
/* bf16 rows of 64s of channels on 16 bytes), for a piece of the classes 8    */
/* bytes a row and 64 classes of statistics (64 MB or 4096 classes) and, with */
/* gradients, 4 or 6 bytes of dz a row and class (512 MB or 2048 classes),    */
/* fp32 sums of dx where there are several pieces, and sums of split products. */
/* ------------------------------------------------------------------------- */
#define PVCONV_CE_MAX_CHANNELS 65536
size_t pvconv_linear_cross_entropy_workspace_size(int M, int K, int V, pvconv_dtype x_dt,
                                                  pvconv_dtype w_dt, pvconv_dtype dx_dt,
                                                  pvconv_dtype dw_dt, int want_grad);
pvconv_status pvconv_linear_cross_entropy(
    const void* x, pvconv_dtype x_dt, int x_ld, const void* w, pvconv_dtype w_dt, int w_ld, int M,
    int K, int V, const float* bias, const int32_t* labels, const float* row_weight, float* loss,
    float* lse, void* dx, pvconv_dtype dx_dt, int dx_ld, void* dw, pvconv_dtype dw_dt,
    float* dbias, void* workspace, size_t workspace_bytes, void* stream);

/* The gradients alone, from the lse of a forward with the same x, w and bias; */
/* dloss [M] fp32 (or NULL: 1) in the place of row_weight.                   */
pvconv_status pvconv_linear_cross_entropy_backward(
    const void* x, pvconv_dtype x_dt, int x_ld, const void* w, pvconv_dtype w_dt, int w_ld, int M,
    int K, int V, const float* bias, const int32_t* labels, const float* lse, const float* dloss,
    void* dx, pvconv_dtype dx_dt, int dx_ld, void* dw, pvconv_dtype dw_dt, float* dbias,
    void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PVCONV_TRAIN_H */
