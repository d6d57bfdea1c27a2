// Declarations shared by the kernels and the C entry points of the local
// models (som_local.h).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace som {

enum : int32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };                       // som_type
enum : int32_t { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };  // som_activation
enum : int32_t { kForward = 0, kInput = 1, kWeight = 2 };               // which product

inline int type_size(int32_t type) { return type == kF32 ? 4 : 2; }

// The activations and their slopes, on the hardware's exponential and reciprocal
// (each within one unit in the last place): an exact division or the library's
// error function would take longer than the products they follow (gelu of
// 8192 x 8192 sums: 110 us of 440).  The normal distribution's tail
//     q = 1 - Phi(|z|) = (a1 t + ... + a5 t^5) e^(-z^2 / 2) / 2,
//     t = 1 / (1 + p |z| / sqrt 2)
// is Abramowitz and Stegun, formula 7.1.26, off by at most 7.5e-8; its exponential
// is the slope's too, and for negative z the tail itself is the value, so nothing
// cancels.
__device__ inline float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

__device__ inline void normal(float z, float *below, float *bell) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.f));
    const float e = exp_fast(-0.5f * z * z);
    float s = fmaf(t, 1.061405429f, -1.453152027f);
    s = fmaf(t, s, 1.421413741f);
    s = fmaf(t, s, -0.284496736f);
    s = fmaf(t, s, 0.254829592f);
    const float tail = 0.5f * t * s * e;
    *below = z > 0.f ? 1.f - tail : tail;
    *bell = e;
}

__device__ inline float sigmoid_fast(float z) {
    return __builtin_amdgcn_rcpf(1.f + exp_fast(-z));
}

__device__ inline float activate(float z, int32_t kind) {
    switch (kind) {
        case kActRelu: return z > 0.f ? z : (z != z ? z : 0.f);
        case kActGelu: {
            float below, bell;
            normal(z, &below, &bell);
            return z * below;
        }
        case kActSilu: return z * sigmoid_fast(z);
        default: return z;
    }
}

__device__ inline float activation_slope(float z, int32_t kind) {
    switch (kind) {
        case kActRelu: return z > 0.f ? 1.f : 0.f;
        case kActGelu: {
            float below, bell;
            normal(z, &below, &bell);
            return fmaf(z * bell, 0.39894228040143268f, below);
        }
        case kActSilu: {
            const float q = sigmoid_fast(z);
            return fmaf(z * q, 1.f - q, q);
        }
        default: return 1.f;
    }
}

// Largest e in [0, experts) whose first tile offsets[e] / tile + e is at most
// t, or with tile = 0 whose first row is at most t: 64 places tested at a time.
// (An expert of c rows from row o on has the tiles from o / tile + e on; the next
// one's begin at least ceil(c / tile) later, and the last ones may be empty.)
__device__ inline int expert_of(const int32_t *offsets, int experts, int tile, int64_t t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, span = experts;
    while (span > 1) {
        const int width = (span + 63) / 64;
        const int e = lo + lane * width;
        const bool at_most = lane * width < span &&
                             (tile ? (int64_t)(offsets[e] / tile) + e : (int64_t)offsets[e]) <= t;
        const int last = 63 - __clzll(__ballot(at_most) | 1);
        lo += last * width;
        span = span - last * width < width ? span - last * width : width;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// The tiles' kernels reach an operand's elements by 32-bit offsets within a tile's
// rows, and within a whole listed matrix (som_product.h).
constexpr int64_t kMaxWidth = 4000000;
inline bool tile_reaches(int64_t ld, int size) { return ld * size * 256 < ((int64_t)1 << 32); }

// C = A B^T, C of m rows and n columns, contraction k (som_product.h).
//   forward  A = x (m x k), B = w (n x k):      y = act(C + bias) + residual
//   input    A = dz (m x k), B = w (k x n):     dx = C [* slope of z]
//   weight   A = dz (k x m), B = x (k x n):     dw = C
// Routed (offsets): forward and input take the m rows by expert, offsets[e] ..
// of B + e batch_b; weight sums offsets[e] .. into dw + e m n.  list: forward,
// row r of A is A's row list[r] / per; weight, row s of B is B's row
// list[s] / per.  Rows past offsets[experts] are not touched.
struct ProductArgs {
    int32_t mode, type, activation;
    const void *a, *b;
    int64_t lda, ldb, batch_b;
    int64_t m, n, k;
    const void *bias, *residual, *slope;
    int64_t ldr;
    void *y, *z;
    const int32_t *offsets, *list;
    int32_t experts, per;
    int32_t splits;       // parts of the contraction
    float *partial;       // splits x partial_rows x whole tiles
    int64_t partial_rows;
};

// How a product runs.
struct ProductPlan {
    int32_t tile;         // rows and columns of a tile: 256, 128 or 64; of few rows, rows: 16
    int32_t waves;        // few rows: waves of a workgroup; otherwise 0
    int32_t splits;       // parts of the contraction
    bool aligned;         // both sides lie in whole 16-byte pieces
    double time;          // estimated microseconds
    int64_t partial_floats;
};

// Copies `rows` rows of `cols` elements, `lds` apart, to rows of ldd >= cols
// elements filled up with zeros; with z (rows ldz apart), times act'(z); with a
// list, row r is src's row list[r] / per, or zeros where list[r] is negative.
struct RowsArgs {
    int32_t type, activation;
    const void *src, *z;
    void *dst;
    int64_t rows, cols, lds, ldz, ldd;
    const int32_t *list;
    int32_t per;
};
hipError_t launch_rows_copy(const RowsArgs &a, hipStream_t stream);

// out[e] = sums of the rows of src (cols elements, ld apart) of expert e, or of all
// rows without offsets.
struct SumsArgs {
    int32_t type;
    const void *src;
    int64_t rows, cols, ld;
    const int32_t *offsets;
    int32_t experts;
    void *out;
    float *partial;         // sums_partial() floats
};
int64_t sums_partial(const SumsArgs &a);
hipError_t launch_sums(const SumsArgs &a, hipStream_t stream);

struct CombineArgs {
    int32_t type, k;
    int64_t n, width;
    const void *y;          // rows in the experts' order
    const float *weight;    // n x k, or null
    const int32_t *place;   // n x k
    const void *residual;   // forward
    int64_t ldr;
    void *out;
    const void *dout;       // backward
    int64_t ldd;
    void *dy, *dweight;
};
hipError_t launch_combine(const CombineArgs &a, hipStream_t stream);
hipError_t launch_combine_backward(const CombineArgs &a, hipStream_t stream);

// som_route.hip; the fields are som_route_call's.
constexpr int kMaxExperts = 16384, kMaxChoices = 64, kMaxGroups = 64;
struct RouteArgs {
    int32_t type, softmax;
    int64_t n;
    int32_t experts, k, groups, top_groups, group_best, renormalise;
    float scale;
    const void *scores;
    int64_t lds;
    const float *bias;
    int32_t *index;
    float *weight;
    const void *dweight;
    int32_t dweight_type;
    void *dscores;
};
hipError_t launch_route(const RouteArgs &a, hipStream_t stream);
hipError_t launch_route_backward(const RouteArgs &a, hipStream_t stream);

struct DispatchArgs {
    const int32_t *index;
    int64_t slots;
    int32_t experts;
    int32_t *offsets, *order, *place;
    int32_t *counts;        // blocks x experts
    int32_t blocks;
};
int32_t dispatch_blocks(int64_t slots);
hipError_t launch_dispatch(const DispatchArgs &a, hipStream_t stream);

// som_adamw.hip
constexpr int kAdamwBlock = 256, kAdamwChunk = 2048, kAdamwGrads = 256;
struct AdamwChunk {         // up to kAdamwChunk elements of one tensor
    int32_t tensor;         // within its launch
    int32_t first;          // first element, in units of kAdamwBlock
};
struct AdamwTensor {
    void *param;
    int64_t count, state;   // elements; where its states begin
    int32_t type, pad;
};
struct AdamwArgs {
    const AdamwChunk *chunks;
    const AdamwTensor *tensors;
    void *mean, *square;
    float *mean_scale, *square_scale, *master;
    float beta1, rest1, beta2, rest2, decay, rate, root_scale, eps;
    int32_t nchunks;
    const void *grads[kAdamwGrads];
    unsigned char grad_type[kAdamwGrads];
};
hipError_t launch_adamw(const AdamwArgs &a, bool eight, hipStream_t stream);

ProductPlan plan_product(const ProductArgs &a, bool aligned, int num_cus);
// One per element type (som_product_*.hip).
hipError_t launch_product_f32(ProductArgs a, const ProductPlan &p, hipStream_t stream);
hipError_t launch_product_bf16(ProductArgs a, const ProductPlan &p, hipStream_t stream);
hipError_t launch_product_f16(ProductArgs a, const ProductPlan &p, hipStream_t stream);

}  // namespace som
