// Declarations shared by the kernels and the C entry points of the local
// models (som_local.h).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace som {

enum : int32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };                       // som_type
enum : int32_t { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };  // som_activation
enum : int32_t { kForward = 0, kInput = 1, kWeight = 2, kGate = 3 };    // which product

inline int type_size(int32_t type) { return type == kF32 ? 4 : 2; }

// A dimension of a grid counts its threads in 32 bits.
inline bool grid_holds(int64_t blocks, int64_t threads) {
    return blocks <= ((int64_t)UINT32_MAX) / threads;
}

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
    const float e = __builtin_amdgcn_exp2f(z * z * (-0.5f * 1.44269504f));
    float s = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
    s = fmaf(t, s, 0.5f * 1.421413741f);
    s = fmaf(t, s, 0.5f * -0.284496736f);
    s = fmaf(t, s, 0.5f * 0.254829592f);
    const float tail = t * s * e;
    *below = z > 0.f ? 1.f - tail : tail;
    *bell = e;
}

__device__ inline float sigmoid_fast(float z) {
    return __builtin_amdgcn_rcpf(1.f + exp_fast(-z));
}

// The activation and, where it is wanted, its slope.
__device__ inline float activate(float z, int32_t kind, float *slope = nullptr) {
    switch (kind) {
        case kActRelu:
            if (slope) *slope = z > 0.f ? 1.f : 0.f;
            return z > 0.f ? z : (z != z ? z : 0.f);
        case kActGelu: {
            float below, bell;
            normal(z, &below, &bell);
            if (slope) *slope = fmaf(z * bell, 0.39894228040143268f, below);
            return z * below;
        }
        case kActSilu: {
            const float q = sigmoid_fast(z);
            if (slope) *slope = fmaf(z * q, 1.f - q, q);
            return z * q;
        }
        default:
            if (slope) *slope = 1.f;
            return z;
    }
}

// N neighbouring values of a row to and from memory, `left` of them there.  Rows
// begin at any element: the hardware takes 16 bytes at any address.
template <typename T, int N>
struct Piece {
    typedef T Vec __attribute__((ext_vector_type(N)));
    Vec v;
    __device__ void read(const T *p, int left) {
        if (left >= N) {
            __builtin_memcpy(&v, __builtin_assume_aligned(p, sizeof(T)), sizeof(Vec));
        } else if (left > 0) {   // without branches, so that the reads are under way together
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const T u = p[e < left ? e : 0];
                v[e] = e < left ? u : (T)0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (T)0.f;
        }
    }
    __device__ void write(T *p, int left) const {
        if (left >= N) {
            __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T)), &v, sizeof(Vec));
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e < left) p[e] = v[e];
        }
    }
};

// Division of whole numbers below 2^31 by one that is not known when compiling: a
// product with a rounded-up reciprocal and a shift.
struct Divider {
    uint32_t by, magic, shift;
    Divider() : by(1), magic(0), shift(0) {}
    explicit Divider(uint32_t d) : by(d), magic(0), shift(0) {
        uint32_t log = 0;
        while ((uint64_t)1 << log < d) ++log;
        if (log == 0) return;
        shift = log - 1;
        magic = (uint32_t)((((uint64_t)1 << (32 + shift)) / d) + 1);
    }
    __device__ uint32_t quotient(uint32_t v) const {
        return magic ? __umulhi(v, magic) >> shift : v;
    }
};

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

// A weight is gate_kept * 2^gate_exponent.  fp16 holds no product of an activation and a
// small weight: what is kept beside the activation is then the weight without its
// power of two (magnitudes of 1/2 to 1; larger weights whole), and the power goes to the
// other factor of the product, a gradient, which a loss scale keeps within the type.
__device__ inline float gate_kept(float g) {
    return fabsf(g) < 0.5f ? __builtin_amdgcn_frexp_mantf(g) : g;
}
__device__ inline int gate_exponent(float g) {
    return fabsf(g) < 0.5f ? __builtin_amdgcn_frexp_expf(g) : 0;
}

// C = A B^T, C of m rows and n columns, contraction k (som_product.h).
//   forward  A = x (m x k), B = w (n x k):      z = C + bias, y = act(z) + residual,
//                                               scaled = gate act(z) (fp16: gate_kept act(z))
//   input    A = dz (m x k), B = w (k x n):     y = C
//   gate     A = dout (m x k), B = w (k x n):   y = gate C act'(argument),
//                                               dots: parts of <C, act(argument)>
//   weight   A = dz (k x m), B = x (k x n):     y = C
// Routed (offsets): the m rows of forward, input and gate lie by expert, offsets[e]
// .. of B + e batch_b; weight sums offsets[e] .. into y + e m n.  Rows past
// offsets[experts] are not touched.  list: row r of A (forward, gate) or row s of B
// or A (weight) is the matrix's row list[.] / per.  slots: the slot of each row.
struct ProductArgs {
    int32_t mode, type, activation;
    int32_t wide;                     // y holds fp32 (not in weight)
    const void *a, *b;
    int64_t lda, ldb, batch_b;
    int64_t m, n, k;
    const void *bias, *residual;
    int64_t ldr;
    void *y, *z, *scaled;
    const int32_t *offsets, *list, *slots;
    int32_t experts, list_of_a;
    Divider per;
    const float *gates;               // by slot; gate: null for 1
    const void *argument;             // gate: rows of n, ld_argument apart
    int64_t ld_argument;
    int32_t argument_listed;          // row r's is the document's, slots[r] / per
    const void *image;                // rows of n: forward's scaled, of act(argument); or null
    float *dots;                      // gate: m x dot_cols
    int32_t dot_cols;
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

// The expert with the `rank`-th most rows (the lower of equals first), of up to 64;
// of more, where the sizes of those that run together even out, expert `rank`.
__device__ inline int expert_of_rank(const int32_t *offsets, int experts, int rank) {
    if (experts > 64) return rank;
    const int lane = threadIdx.x & 63;
    const int rows = lane < experts ? offsets[lane + 1] - offsets[lane] : -1;
    int before = 0;
    for (int e = 0; e < experts; ++e) {
        const int other = __builtin_amdgcn_readlane(rows, e);
        before += other > rows || (other == rows && e < lane) ? 1 : 0;
    }
    const unsigned long long who = __ballot(lane < experts && before == rank);
    return __builtin_amdgcn_readfirstlane(__ffsll((long long)who) - 1);
}

// Copies `rows` rows of `cols` elements, `lds` apart, to rows of ldd >= cols
// elements filled up with zeros; with z (rows ldz apart), times act'(z); with a
// list, row r is src's row list[r] / per, or zeros where list[r] is negative, times
// gates[list[r]], or their powers of two alone (gate_exponent), if there are any.
struct RowsArgs {
    int32_t type, activation;
    const void *src, *z;
    void *dst;
    int64_t rows, cols, lds, ldz, ldd;
    const int32_t *list;
    Divider per;
    const float *gates;     // times gates[list[r]]
    int32_t exponents;      // the gates' powers of two alone
    Divider pieces;         // of a row of dst
};
hipError_t launch_rows_copy(const RowsArgs &a, hipStream_t stream);

// out[e] = sums of the rows of src (cols elements, ld apart) of expert e, or of all
// rows without offsets.  With a list, row r is src's row list[r] / per times
// gates[list[r]], and dots holds the parts of <src's row, bias of the row's expert>:
// rows x dot_cols.
struct SumsArgs {
    int32_t type;
    const void *src;
    int64_t rows, cols, ld;
    const int32_t *offsets;
    int32_t experts;
    const int32_t *list;
    Divider per;
    const float *gates;
    const void *bias;
    float *dots;
    int32_t dot_cols;
    void *out;              // null: dots alone
    float *partial;         // sums_partial() floats
};
int32_t sums_dot_cols(const SumsArgs &a);
int64_t sums_partial(const SumsArgs &a);
hipError_t launch_sums(const SumsArgs &a, hipStream_t stream);

// out[i] = residual[i] + sum over j of weight[i][j] y[place[i][j]], y in fp32.
struct CombineArgs {
    int32_t type, k;
    int64_t n, width;
    const float *y;         // rows in the experts' order
    const float *weight;    // n x k, or null
    const int32_t *place;   // n x k
    const void *residual;
    int64_t ldr;
    void *out;
    Divider pieces;         // of a row of out
};
hipError_t launch_combine(const CombineArgs &a, hipStream_t stream);

// dweight[s] = sums of the parts of row place[s] in both arrays (0 if absent).
struct DweightArgs {
    int32_t type;
    int64_t slots;
    const int32_t *place;
    const float *dots[2];
    int32_t cols[2];
    void *dweight;
};
hipError_t launch_dweight(const DweightArgs &a, hipStream_t stream);

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
hipError_t launch_route_backward(const RouteArgs &a, hipStream_t stream);

struct DispatchArgs {
    const int32_t *index;
    int64_t slots;
    int32_t experts;
    int32_t *offsets, *order, *place;
    int32_t *counts;        // (blocks + 1) x experts
    int32_t blocks, scanned;
};
int32_t dispatch_blocks(int64_t slots);
hipError_t launch_dispatch(const DispatchArgs &a, hipStream_t stream);
// Whether the routing's kernel can sort its slots too (few, in one workgroup), and
// the routing, with that sort if it is given.
bool route_sorts(const RouteArgs &a);
hipError_t launch_route(const RouteArgs &a, const DispatchArgs *sort, hipStream_t stream);

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
// Parts of a row's dots: columns of one wave each.
inline int32_t plan_dot_cols(const ProductPlan &p, int64_t n) {
    const int64_t wide = p.tile == 64 ? 32 : 64;
    return (int32_t)((n + wide - 1) / wide);
}
// One per element type (som_product_*.hip).
hipError_t launch_product_f32(ProductArgs a, const ProductPlan &p, hipStream_t stream);
hipError_t launch_product_bf16(ProductArgs a, const ProductPlan &p, hipStream_t stream);
hipError_t launch_product_f16(ProductArgs a, const ProductPlan &p, hipStream_t stream);

}  // namespace som
