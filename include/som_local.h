/*
 * som_local.h -- C ABI of libsom for local models on a trained map: a gate that
 * sends each document to a few experts (for example the units of a map), the
 * experts' matrix products, their gradients, and the optimizer that trains
 * both.
 *
 * With prototypes w_u, the scores -|x - w_u|^2 / (2 tau) of a document x are, up
 * to a constant per document, x . (w_u / tau) - |w_u|^2 / (2 tau): one product with
 * a bias (som_linear).  The k best of them and their softmax (som_route) are a
 * soft form of the map's best-matching units; with k = 1 the BMU itself.  Each
 * document is then answered by its experts (som_experts).
 *
 * Conventions shared with som.h: every call returns a som_status, none throws
 * or aborts; arguments are validated before any device work; device pointers
 * are checked against their allocations (best effort under a pooling
 * allocator) and stay the caller's; calls are ordered on the `stream` they are
 * given (a hipStream_t, NULL for the null stream), return after enqueueing,
 * and can be captured into a graph.  Calls keep no state of their own: work
 * memory is the caller's (som_*_workspace say how much), must be 256-byte
 * aligned, and may be reused once the stream has passed the call.
 * Calls on different streams and host threads are independent.
 *
 * Matrices are row-major; "packed" means that rows follow each other without
 * a gap.  Sums are fp32 whatever the element type and are rounded once, when a
 * result is stored.  NaN and infinities in the data propagate as in IEEE
 * arithmetic; nothing is scanned.
 */
#ifndef SOM_LOCAL_H
#define SOM_LOCAL_H

#include "som.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the matrices. */
typedef enum som_type { SOM_F32 = 0, SOM_BF16 = 1, SOM_F16 = 2 } som_type;

/* NONE z;  RELU max(z, 0);  GELU z (1 + erf(z / sqrt 2)) / 2;  SILU z / (1 + e^-z). */
typedef enum som_activation {
    SOM_ACT_NONE = 0, SOM_ACT_RELU = 1, SOM_ACT_GELU = 2, SOM_ACT_SILU = 3
} som_activation;

/* A product with its epilogue,
 *     z = x w^T + bias,    y = act(z) + residual,
 * of x (n x inner) and w (outer x inner).
 *
 * Gradients (som_linear_backward), from dy, with dz = dy act'(z):
 *     dx = dz w    dw = dz^T x    dbias = sum of dz's rows
 * The residual's gradient is dy itself.  With an activation, dz is held in the
 * element type, as the matrix instructions take it, for the two products and dbias.
 *
 * Written for an activation, z keeps finite sums finite where the type would round
 * them to infinity, and relu's positive ones above 0 where it would round them to 0.
 * relu's slope is that of the fp32 sum's sign.  A sum of K products
 * is off by up to about K 2^-24 of their magnitudes: where z in exact arithmetic
 * is nearer to 0 than that, its slope can be 1 or 0, and such an element's whole part
 * of the gradients is there or not (of sums of 2000 products about one sign in 16
 * million is unlike the exact one).  som_experts' first layer is no different. */
typedef struct som_linear_call {
    int32_t type;              /* som_type of all matrices                           */
    int32_t activation;        /* som_activation                                     */
    int64_t n;                 /* rows (documents); 0 is allowed                     */
    int32_t inner, outer;      /* 1 .. 4,000,000                                     */
    const void *x;
    int64_t ldx;               /* elements from row to row, >= inner                 */
    const void *w;             /* packed outer x inner                               */
    const void *bias;          /* outer; NULL for none                               */
    const void *residual;      /* NULL for none (forward only)                       */
    int64_t ldr;               /* >= outer                                           */
    void *y;                   /* packed, forward's result                           */
    void *z;                   /* packed; forward writes it unless NULL; backward
                                  reads it unless activation is NONE               */
    const void *dy;            /* backward                                           */
    int64_t lddy;              /* >= outer                                           */
    void *dx, *dw, *dbias;     /* packed; each NULL if not wanted                    */
    void *workspace;
    uint64_t workspace_bytes;
    void *stream;
} som_linear_call;

/* Bytes of work memory that the call needs (0: none, workspace may be NULL):
 * parts of a split contraction or of sums, copies of operands whose rows are not
 * whole 16-byte pieces where that is the faster way, and dz.  A function of the
 * sizes, leading dimensions, pointer alignments and which pointers are NULL. */
som_status som_linear_workspace(const som_linear_call *call, int32_t backward, uint64_t *bytes);

/* How the call's products run, in the order y; dx, dw: the rows and columns of a
 * workgroup's tile (256, 128 or 64; 16: the kernel of few rows), negative where its
 * operands go through registers and not straight into LDS, 0 for a product that the
 * call does not have.  A function of the same things as the work memory. */
som_status som_linear_route(const som_linear_call *call, int32_t backward, int32_t tiles[2]);

/* Errors of both: SOM_E_ARG (a bad type, activation or size, a missing or too
 * short array, a leading dimension below its row, a workspace that is missing,
 * misaligned or too small), SOM_E_UNSUPPORTED (inner or outer above 4,000,000;
 * results of 2^36 elements, the columns counted in whole 64s), SOM_E_DEVICE. */
som_status som_linear(const som_linear_call *call);
som_status som_linear_backward(const som_linear_call *call);

/* The experts' answers to the documents x (n x inner) that are routed to them,
 * joined: for document i with experts e = index[i][j] and weights g = weight[i][j],
 *     z = w1_e x_i + b1_e,   h = act(z),   answer = w2_e h + b2_e,
 *     y_i = residual_i + sum over j of g answer,
 * or, with w2 NULL, local linear maps: answer = w1_e x_i + b1_e (activation NONE).
 * The routing comes as som_dispatch gives it; a slot whose expert is -1 adds
 * nothing, unless its weight is NaN: then the document's y is NaN.
 *
 * For a gradient, forward has to keep z and scaled = g h (both n k x hidden,
 * rows in the experts' order; without w2 nothing is kept).  In fp16, which does not
 * hold small products, scaled is that of g / 2^e with |g| / 2^e in [1/2, 1) where
 * |g| < 1/2, and the gradient takes 2^e dy.  From dy,
 *     dweight = <dy_i, answer>  (of the element type; 0 for absent slots)
 *     dz = g (w2_e^T dy_i) act'(z)
 *     dw2_e = sum of dy_i scaled^T,  db2_e = sum of g dy_i
 *     dw1_e = sum of dz x_i^T,  db1_e = sum of dz,  dx_i = sum over j of w1_e^T dz
 * An expert without documents gets zeros.  The residual's gradient is dy.
 * Rounded to the element type on the way: h (scaled apart, from the same sums), z
 * where the slope is taken of it, dz, without w2 g dy_i for dw1; answers and each slot's part of dx are joined
 * in fp32.  dweight is formed as <w2_e^T dy_i, h> + <dy_i, b2_e> with h, in 16-bit
 * types, the mean of act(z) and scaled / g (its part of g). */
typedef struct som_experts_call {
    int32_t type;              /* som_type of all matrices                           */
    int32_t activation;        /* som_activation                                     */
    int64_t n;                 /* documents; 0 is allowed                            */
    int32_t k, experts;        /* choices of a document, n k <= 2^31 - 1; 1 .. 16384 */
    int32_t inner, hidden;     /* 1 .. 4,000,000; x's width, w1's rows               */
    int32_t outer;             /* w2's rows; without w2 equal to hidden              */
    const void *x;
    int64_t ldx;
    const void *w1, *b1;       /* packed experts x hidden x inner, experts x hidden  */
    const void *w2, *b2;       /* packed experts x outer x hidden, experts x outer;
                                  a bias NULL for none                               */
    const void *residual;      /* n x outer, NULL for none (forward only)            */
    int64_t ldr;
    const float *weight;       /* n x k; NULL for 1                                  */
    const int32_t *offsets, *order, *place;  /* som_dispatch's                       */
    void *y;                   /* packed n x outer                                   */
    void *z, *scaled;          /* kept for the gradient; forward: both or neither    */
    const void *dy;            /* n x outer, backward                                */
    int64_t lddy;
    void *dx;                  /* packed n x inner; each gradient NULL if not wanted */
    void *dweight;             /* packed n x k                                       */
    void *dw1, *db1, *dw2, *db2;
    void *workspace;
    uint64_t workspace_bytes;
    void *stream;
} som_experts_call;

/* Errors: as som_linear, and SOM_E_ARG (b2 without w2, an activation, kept arrays
 * or another outer without w2, only one of z and scaled), SOM_E_UNSUPPORTED (more
 * than 16384 experts, n k or experts times hidden or outer above 2^31 - 1). */
som_status som_experts_workspace(const som_experts_call *call, int32_t backward,
                                 uint64_t *bytes);
/* As som_linear_route, in the order w1's, w2's;  dy w2 (dy w1 without w2), its
 * matrix's gradient, dz w1, dw1. */
som_status som_experts_route(const som_experts_call *call, int32_t backward, int32_t tiles[4]);
som_status som_experts(const som_experts_call *call);
som_status som_experts_backward(const som_experts_call *call);

/* Routing of n documents by their scores s (n x experts) to k experts each.
 *     p = softmax(s) over the row, or 1 / (1 + e^-s)
 *     v = s + bias (softmax)  or  p + bias (sigmoid)
 * An expert is closed to a document where s or v is -infinity or NaN.  With
 * groups > 1 the experts form `groups` equal groups of neighbours; a group's
 * value is the sum of its group_best (1 or 2) largest open v (fp32's lowest
 * value where that is below it), and the
 * top_groups groups of the largest values stay, the others' experts are closed
 * too.  index[i][j] is the expert with the j-th largest v left (the lowest index
 * among equals), -1 where none is left.  The bias, one fp32 per expert, acts on
 * the choice alone:
 *     weight[i][j] = scale p[index]            (0 for -1), or, renormalised,
 *     weight[i][j] = scale p[index] / sum over the row's chosen p   (0 if that is 0).
 * (In softmax mode the bias is added to the scores: p + bias would make the
 * choice between near equals depend on the rounding of the row's sum.)
 * A row that holds a NaN (softmax: or +infinity) gets index -1 and weight NaN
 * throughout; a row without an open expert index -1 and weight 0. */
typedef enum som_gate { SOM_GATE_SOFTMAX = 0, SOM_GATE_SIGMOID = 1 } som_gate;

typedef struct som_route_call {
    int32_t type;              /* som_type of scores and dscores                     */
    int32_t gate;              /* som_gate                                           */
    int64_t n;
    int32_t experts;           /* 1 .. 16384                                         */
    int32_t k;                 /* 1 .. min(experts, 64)                              */
    int32_t groups;            /* divides experts, <= 64; 1 for none                 */
    int32_t top_groups;        /* 1 .. groups                                        */
    int32_t group_best;        /* 1 or 2                                             */
    int32_t renormalise;
    float scale;
    const void *scores;
    int64_t lds;               /* elements from row to row, >= experts               */
    const float *bias;         /* NULL for none; finite or -infinity                 */
    int32_t *index;            /* n x k, packed: written by som_route                */
    float *weight;             /* n x k, packed: written by som_route                */
    const void *dweight;       /* n x k, packed                                      */
    int32_t dweight_type;      /* som_type                                           */
    void *dscores;             /* n x experts, packed                                */
    int32_t *offsets;          /* NULL, or with order and place: as som_dispatch     */
    int32_t *order, *place;
    void *workspace;           /* som_dispatch_workspace bytes                       */
    uint64_t workspace_bytes;
    void *stream;
} som_route_call;

/* Errors of both: SOM_E_ARG, SOM_E_UNSUPPORTED (n k above 2^31 - 1), SOM_E_DEVICE.
 * The gradient treats index as given; of a row with weight NaN it is NaN. */
som_status som_route(const som_route_call *call);
som_status som_route_backward(const som_route_call *call);

/* The slots i k + j of an assignment index (n x k, entries in [0, experts) or -1
 * for absent; others count as absent) in the order of their experts, within an
 * expert in their own order: order[p] is the slot of row p, place[i k + j] the row
 * of a slot (-1 if absent), offsets[e] the first row of expert e (experts + 1
 * entries).  order's rows from offsets[experts] on are -1.  n k <= 2^31 - 1.
 * work: som_dispatch_workspace bytes (0: NULL is allowed). */
som_status som_dispatch_workspace(int64_t n, int32_t k, int32_t experts, uint64_t *bytes);
som_status som_dispatch(const int32_t *index, int64_t n, int32_t k, int32_t experts,
                        int32_t *offsets, int32_t *order, int32_t *place, void *work,
                        uint64_t work_bytes, void *stream);

/* AdamW over many tensors at once.  Step t of element p with gradient g:
 *     m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
 *     p = p (1 - lr weight_decay)
 *         - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * in fp32 without contraction into fused operations.  The states of all
 * tensors lie in one array each, tensor i from the next multiple of 256
 * elements on (som_adamw_room elements in all; what lies between tensors is
 * not touched).  With bits = 32 they are fp32 m and v.  With bits = 8 they are e4m3
 * codes (OCP: 448 the largest) of m and of sqrt(v) in units of one fp32 scale per
 * 256 elements, the largest magnitude (at least 1e-30) / 448; a sqrt(v) above 0
 * is never held as 0, so that no step divides by eps alone.  The step
 * itself uses the new m and v before they are rounded.  With master the
 * parameters are kept in fp32 there and `param` is their rounding; without,
 * `param` itself is updated and rounded. */
typedef struct som_adamw_tensor {
    void *param;               /* packed, device                                     */
    int64_t count;             /* elements, >= 0                                     */
    int32_t type;              /* som_type                                           */
} som_adamw_tensor;

typedef struct som_adamw som_adamw;

int64_t som_adamw_room(const som_adamw_tensor *tensors, int32_t count);

/* mean, square: the state arrays; mean_scale, square_scale: room / 256 floats (bits
 * = 8, otherwise NULL); master: room floats or NULL.  All stay the caller's and
 * are used by every later step.  The optimizer keeps a table of 16 bytes per
 * 2048 elements on the current device.  Synchronizes the device.
 * Errors: SOM_E_ARG, SOM_E_OOM, SOM_E_DEVICE. */
som_status som_adamw_create(const som_adamw_tensor *tensors, int32_t count, int32_t bits,
                            void *mean, void *square, float *mean_scale, float *square_scale,
                            float *master, som_adamw **out);
som_status som_adamw_destroy(som_adamw *opt);

/* One step, number `step` (1 for the first), with grads[i] the packed gradient of
 * tensor i, of grad_types[i].  The arrays themselves are host memory, read
 * before the call returns.
 * Errors: SOM_E_ARG (NULLs, step < 1, lr, eps or weight_decay negative or not
 * finite, a beta outside [0, 1), a gradient that does not cover its tensor),
 * SOM_E_DEVICE. */
som_status som_adamw_step(som_adamw *opt, const void *const *grads, const int32_t *grad_types,
                          int64_t step, double lr, double beta1, double beta2, double eps,
                          double weight_decay, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SOM_LOCAL_H */
