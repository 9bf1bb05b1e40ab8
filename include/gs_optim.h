/*
 * gs_optim.h - the optimiser step of a training iteration (the paper trains
 * with Adam, Sec. 6, one learning rate per kind of parameter): AdamW over
 * many tensors in one launch, with moments in 32 or in 8 bits, the global
 * gradient norm with clipping, and the moments carried through a
 * densification. Same library and conventions as gs.h: device pointers the
 * caller owns, work enqueued on the caller's stream (nothing here waits),
 * gs_status codes with gs_last_error(), no device memory allocated by the
 * library. Every call may be captured into a HIP graph.
 *
 * The update of one parameter, in float32, at step t = 1, 2, ... (lr' = lr
 * lr_scale; the 1 / (1 - beta^t) terms and 1 - beta are formed in float64
 * and rounded once; g' = clip g; products and sums round once each or are
 * fused, root and reciprocal are good to an ulp):
 *   m <- beta1 m + (1 - beta1) g'
 *   v <- beta2 v + ((1 - beta2) g') g'
 *   p <- p - ( lr' / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)  +  lr wd lr_scale p )
 * The two terms are added before they leave p: a factor 1 - lr wd would lose
 * most of a small decay to its own rounding. lr wd lr_scale is formed as
 * (lr lr_scale) wd. weight_decay = 0 gives Adam.
 *
 * 8-bit moments are MXFP8 blocks: m, and s = sqrt(v) in v's place, as OCP
 * E4M3 values with one E8M0 scale 2^e per 32 consecutive elements of the
 * tensor (the last block may be shorter). e is the smallest exponent >= -126
 * with |x| <= 448 2^e for the block's finite values, so nothing saturates.
 * The update reads v = s s, is formed in float32 as above, and p is updated
 * from the unrounded m and v; then m and s are rounded to the block's grid,
 * up with probability equal to the share of the way ((k + 1/2) / 2^16 with
 * 16 random bits k). Rounding to the nearest would not do: with 1 - beta2 =
 * 0.001 a falling s moves by a hundredth of the grid's spacing a step, and
 * would never leave its place. A positive s is never rounded to 0 (it becomes
 * the smallest value of its block's grid), so that a remembered m is not
 * divided by a forgotten v. What float32 itself forgets is forgotten: s s is 0
 * for an s of 2^-75 or less, far below any eps in use. Values that are not
 * finite are kept as NaN. All-zero bytes are the state of a new tensor.
 *
 * bfloat16 parameters are rounded up or down with the same kind of odds (16
 * random bits), since most updates are below half their spacing.
 *
 * The random bits of an element are a function of (seed, t, the tensor's
 * place in the list, the element's index) alone, so the same calls give
 * bit-identical results. With mix(x), an integer hash of low bias that
 * C. Wellons published (32 bits): x ^= x >> 16, x *= 0x7feb352d,
 * x ^= x >> 15, x *= 0x846ca68b, x ^= x >> 16:
 *   key  = mix(place + 0x9e3779b9), then key = mix(key ^ w) for w = t's low
 *          and high words, seed's low and high words, the index's high word
 *   bits = mix(index's low word ^ key)
 * m takes the low 16 bits, s the high 16, a bfloat16 parameter the high 16
 * of 0x9e3779b1 * bits.
 */
#ifndef GS_OPTIM_H
#define GS_OPTIM_H

#include "gs.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of parameters and gradients, and the forms of the moments. */
enum { GS_TYPE_F32 = 0, GS_TYPE_BF16 = 1 };
enum { GS_MOMENTS_F32 = 0, GS_MOMENTS_MXFP8 = 1 };

/* A tensor of the list: n contiguous elements. Parameters are float32 with
 * float32 or bfloat16 gradients, or bfloat16 with bfloat16 gradients; the
 * types and moments may differ between the tensors of a list. m and v are
 * float32 arrays [n], or byte arrays [n] with scales [(n + 31) / 32] for
 * MXFP8 moments. Arrays may start at any element. param may be null for a
 * tensor that only counts for gs_grad_norm (of parameters that are held as
 * they are, say): gs_adamw passes it by. Arrays do not overlap. */
typedef struct gs_adamw_tensor {
    void *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale; /* MXFP8 moments only */
    int64_t n;                  /* 0 <= n < 2^40 */
    int32_t param_type, grad_type;
    int32_t moments;
    float lr, weight_decay; /* finite, >= 0 */
} gs_adamw_tensor;

/* The list laid out on the device: the caller fills the buffer fields,
 * gs_plan_adamw the rest. */
typedef struct gs_adamw_plan {
    void *work; /* gs_adamw_plan_bytes() bytes, 256-byte aligned; kept while the plan is in use */
    size_t work_bytes;
    /* filled by gs_plan_adamw */
    int64_t n_items;      /* pieces that the tensors are cut into for the step */
    int64_t n_norm_items; /* and for the norm */
    int64_t step_bytes;   /* what a step reads and writes */
    int64_t norm_bytes;   /* what the norm reads */
    int32_t count;        /* tensors */
    int32_t updatable;    /* whether a tensor with elements has a parameter, or none has elements */
} gs_adamw_plan;

/* What a training run keeps on the device between steps: 64 bytes, 8-byte
 * aligned, zeroed by the caller before the first. */
typedef struct gs_adamw_control {
    int64_t step;    /* updates opened so far: t */
    int64_t skipped; /* calls whose norm was not finite */
    float norm;      /* the last call's norm */
    float clip;      /* the factor of the gradients */
    float first;     /* 1 / (1 - beta1^t) */
    float second;    /* 1 / sqrt(1 - beta2^t) */
    uint32_t apply;  /* whether the last call opened a step */
    uint32_t reserved[7];
} gs_adamw_control;

/* Settings of a step. 0 <= beta < 1, eps >= 2^-126 (an element that never
 * had a gradient is divided by it), lr_scale >= 0 (a schedule's
 * factor on every tensor's learning rate), max_norm > 0 (infinity: no
 * clipping); eps and lr_scale finite as float32 numbers. */
typedef struct gs_adamw_params {
    double beta1, beta2;
    double eps;
    double lr_scale;
    double max_norm;
    uint64_t seed;
} gs_adamw_params;

/* Bytes of plan workspace for a list (-1 cast to size_t for a malformed one:
 * a null list with count > 0, count outside [0, 2^20], a size out of range,
 * or more than 2^31 pieces). */
size_t gs_adamw_plan_bytes(const gs_adamw_tensor *tensors, int64_t count);

/*
 * Lays a list out for gs_grad_norm and gs_adamw. The host array is read
 * before the call returns; the plan holds the arrays' addresses, learning
 * rates and decays, so it is made again when one of these changes (lr_scale
 * changes all rates without that), and kept as long as none does. Work of a plan: calls that share one follow each
 * other.
 */
gs_status gs_plan_adamw(const gs_adamw_tensor *tensors, int64_t count, gs_adamw_plan *plan, hipStream_t stream);

/*
 * The global norm sqrt(sum g^2) of all gradients of the plan, which opens a
 * step of the control: if the sum is finite, t grows by one, clip =
 * max_norm / norm where norm > max_norm and 1 elsewhere, and the
 * bias corrections of the new t are set; otherwise the step is skipped:
 * skipped grows by one and a gs_adamw with this control changes nothing. Sums
 * in float64 in an order that depends on the plan alone: bit-identical
 * between calls. Only beta1, beta2 and max_norm of the settings are used;
 * give gs_adamw the same beta1 and beta2: the corrections left here are of
 * these, the averages of its own.
 */
gs_status gs_grad_norm(const gs_adamw_plan *plan, const gs_adamw_params *params, gs_adamw_control *control,
                       hipStream_t stream);

/*
 * One step of all tensors of the plan that have a parameter (a plan whose
 * tensors all have none is refused). With a control (device memory), t,
 * the clip factor and whether to do anything are what the last gs_grad_norm
 * left there, and step is ignored; with a null control t = step >= 1 and
 * the gradients are taken as they are. A gradient that is not finite makes
 * its own element not finite. Elements are independent (but for the scale of
 * an MXFP8 block), so the result does not depend on how a list is cut or
 * aligned.
 */
gs_status gs_adamw(const gs_adamw_plan *plan, const gs_adamw_params *params, int64_t step,
                   const gs_adamw_control *control, hipStream_t stream);

/* The moments of one array of per-Gaussian parameters: rows of `width`
 * elements (1 .. 64), input and output of the same form. */
typedef struct gs_adamw_rows {
    const void *m, *v;
    const uint8_t *m_scale, *v_scale; /* MXFP8 moments only */
    void *m_out, *v_out;
    uint8_t *m_scale_out, *v_scale_out; /* MXFP8 moments only */
    int32_t width;
    int32_t moments;
} gs_adamw_rows;

#define GS_ADAMW_ROWS_MAX 16

/*
 * Moments through gs_densify's source map: row j of every output array,
 * 0 <= j < n_out, is row source[j] of its input, or 0 where source[j] is
 * negative or not below n_in (a new Gaussian starts with no moments). MXFP8
 * moments fall into new blocks and get new scales by the same rule; values
 * are rounded to the nearest, ties to even (a positive s stays positive).
 * Outputs hold n_out rows and do not overlap the inputs. count is at most
 * GS_ADAMW_ROWS_MAX; 0 <= n_in, n_out < 2^31.
 */
gs_status gs_adamw_carry(const gs_adamw_rows *arrays, int32_t count, int64_t n_in, const int32_t *source,
                         int64_t n_out, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GS_OPTIM_H */
