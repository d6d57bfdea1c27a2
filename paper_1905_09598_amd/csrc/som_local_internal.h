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

__device__ inline float activate(float z, int32_t kind) {
    switch (kind) {
        case kActRelu: return z > 0.f ? z : (z != z ? z : 0.f);
        case kActGelu: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        case kActSilu: return z / (1.f + expf(-z));
        default: return z;
    }
}

__device__ inline float activation_slope(float z, int32_t kind) {
    switch (kind) {
        case kActRelu: return z > 0.f ? 1.f : 0.f;
        case kActGelu:
            return 0.5f * (1.f + erff(z * 0.70710678118654752f)) +
                   z * expf(-0.5f * z * z) * 0.39894228040143268f;
        case kActSilu: {
            const float q = 1.f / (1.f + expf(-z));
            return q * (1.f + z * (1.f - q));
        }
        default: return 1.f;
    }
}

// Which of a product's arrays can be reached four elements at a time.
enum : int32_t { kVecOut = 1, kVecBias = 2, kVecResidual = 4, kVecSlope = 8 };

// C = A B^T, C of m rows and n columns, contraction k (som_product.h).
//   forward  A = x (m x k), B = w (n x k):      y = act(C + bias) + residual
//   input    A = dz (m x k), B = w (k x n):     dx = C [* slope of z]
//   weight   A = dz (k x m), B = x (k x n):     dw = C, bias_grad = sums of dz
// Routed (offsets): forward and input take the m rows by expert, offsets[e] ..
// of B + e batch_b; weight sums offsets[e] .. into dw + e m n.  list: forward,
// row r of A is A's row list[r] / per; weight, row s of B is B's row
// list[s] / per.  Rows past offsets[experts] are not touched.
struct ProductArgs {
    int32_t mode, type, activation, vec;
    const void *a, *b;
    int64_t lda, ldb, batch_b;
    int64_t m, n, k;
    const void *bias, *residual, *slope;
    int64_t ldr;
    void *y, *z, *bias_grad;
    const int32_t *offsets, *list;
    int32_t experts, per;
    int32_t splits;       // parts of the contraction
    float *partial;       // splits x partial_rows x whole tiles, then splits x partial_rows
    int64_t partial_rows;
};

// How a product runs.
struct ProductPlan {
    int32_t tile;         // rows and columns of a tile: 256, 128 or 64; of few rows, rows: 16 or 64
    int32_t waves;        // few rows: waves of a workgroup; otherwise 0
    int32_t splits;       // parts of the contraction
    bool aligned;         // few rows: both sides lie in whole 16-byte pieces
    int64_t partial_floats;
};

// Copies `rows` rows of `cols` elements, `lds` apart, to rows of ldd >= cols
// elements filled up with zeros; with z (rows ldz apart), times act'(z).
struct RowsArgs {
    int32_t type, activation;
    const void *src, *z;
    void *dst;
    int64_t rows, cols, lds, ldz, ldd;
};
hipError_t launch_rows_copy(const RowsArgs &a, hipStream_t stream);

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

ProductPlan plan_product(const ProductArgs &a, int num_cus);
// One per element type (som_product_*.hip).
hipError_t launch_product_f32(ProductArgs a, const ProductPlan &p, hipStream_t stream);
hipError_t launch_product_bf16(ProductArgs a, const ProductPlan &p, hipStream_t stream);
hipError_t launch_product_f16(ProductArgs a, const ProductPlan &p, hipStream_t stream);

}  // namespace som
