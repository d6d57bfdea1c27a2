// Matrix products of the local models on the matrix cores: y = act(x w^T + b)
// + r, its gradients dx = dz w and dw = dz^T x, dense or for the rows of each
// expert.  Included by one translation unit per element type.
//
// One product C = A B^T over a contraction of length k, C's rows from side A,
// its columns from side B.  A side lies in memory either with the contraction
// along its rows ("along": x and w of the forward product, dz of dx) or with one
// row per contraction step ("across": w of dx, dz and x of dw).  Both are read
// from where they lie: nothing is transposed in memory.
//
// A workgroup forms a TM x TN tile in slabs of 128 bytes of contraction (64
// elements of 16 bits, 32 floats).  A slab goes from memory straight into LDS
// (16 bytes a lane), the next one while this one is multiplied, and is read
// back as the 16-byte fragments of the 16 x 16 instructions: side B first, so
// that a lane ends up with four neighbouring columns of one row of C.  Sums
// are fp32 from the first product to the epilogue, which rounds once.
//
// LDS layouts (the writes of one load are contiguous, so the order is made by
// choosing each lane's source):
//   along   row r holds its eight 16-byte pieces in the order c ^ (r & 7): the 16
//           rows of a fragment then lie on all banks.
//   across  contraction step s holds its columns in units of 16, in the order
//           u ^ f(s): the steps that are read together lie on different banks.
//           16-bit types are transposed by the reading instruction.
// Rows beyond C are read from its last row and not stored; the contraction is
// filled up from 16 bytes of zeros.
#pragma once

#include "som_local_internal.h"

#include <algorithm>

namespace som {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;
typedef __attribute__((address_space(3))) s4 *LdsS4;

__device__ const i4 kZeros = {0, 0, 0, 0};

template <typename T>
__device__ inline f4 multiply(i4 b, i4 a, f4 c);

template <>
__device__ inline f4 multiply<__bf16>(i4 b, i4 a, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, b),
                                                   __builtin_bit_cast(b8, a), c, 0, 0, 0);
}
template <>
__device__ inline f4 multiply<_Float16>(i4 b, i4 a, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, b),
                                                  __builtin_bit_cast(h8, a), c, 0, 0, 0);
}
// Four steps of four: which four contraction indices form a step does not
// matter as long as both sides take the same.
template <>
__device__ inline f4 multiply<float>(i4 b, i4 a, f4 c) {
    const f4 bf = __builtin_bit_cast(f4, b), af = __builtin_bit_cast(f4, a);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(bf[j], af[j], c, 0, 0, 0);
    return c;
}

// ---------------------------------------------------------------- one side
// ROWS rows (or columns) of a tile, loaded by WAVES waves.
template <typename T, bool ACROSS, int ROWS, int WAVES>
struct Side {
    static constexpr int kElems = 16 / sizeof(T);           // elements of a 16-byte piece
    static constexpr int kSlab = 128 / sizeof(T);           // contraction of a slab
    static constexpr int kLoads = ROWS / 8 / WAVES;         // 1 KB each, per wave
    static constexpr int kPieces = ROWS / kElems;           // across: pieces of a step
    static constexpr int kUnits = ROWS / 16;                // across: units of 16 columns
    static constexpr int kUnitPieces = 16 / kElems;
    static_assert(kLoads * WAVES * 8 == ROWS, "whole loads");

    const char *src[kLoads];  // this lane's source of the next slab, by load
    int64_t at[kLoads];       // its contraction index there
    int64_t step;             // bytes from slab to slab

    // What the units of contraction step s are exchanged with.
    static __device__ int twist(int s) {
        const int f = sizeof(T) == 2 ? (s & 3) | ((s >> 3) & 1) << 2 : (s >> 2) & 3;
        return f & (kUnits - 1);
    }

    // Rows row0 .. of a side of `rows` rows whose element (r, c) is p[r * ld + c]
    // (along), or columns row0 .. of one whose element is p[c * ld + r]
    // (across); `list`: row r is the side's row list[r] / per.  k0: where the
    // contraction begins, counted from p.
    __device__ void begin(const void *p, int64_t ld, int64_t row0, int64_t rows, int64_t k0,
                          const int32_t *list, int per) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int q = (wave * kLoads + j) * 64 + lane;  // 16-byte place in the LDS slab
            const char *base = static_cast<const char *>(p);
            if (ACROSS) {
                const int s = q / kPieces, place = q % kPieces;
                const int unit = (place / kUnitPieces) ^ twist(s);
                const int64_t c = row0 + unit * 16 + (place % kUnitPieces) * kElems;
                const int64_t col = c < rows ? c : (rows - 1) / kElems * kElems;
                at[j] = k0 + s;
                src[j] = base + ((at[j] * ld) + col) * (int64_t)sizeof(T);
            } else {
                const int r = q >> 3, piece = (q & 7) ^ (r & 7);
                int64_t row = row0 + r < rows ? row0 + r : rows - 1;
                if (list) row = list[row] / per;
                at[j] = k0 + piece * kElems;
                src[j] = base + (row * ld + at[j]) * (int64_t)sizeof(T);
            }
        }
        step = ACROSS ? kSlab * ld * (int64_t)sizeof(T) : 128;
    }

    // Load the next slab into `lds`; contraction indices from k_end on are zeros.
    __device__ void load(char *lds, int64_t k_end, bool whole) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const char *from = src[j];
            if (!whole && at[j] >= k_end) from = reinterpret_cast<const char *>(&kZeros);
            __builtin_amdgcn_global_load_lds((GlobalPtr)from,
                                             (LdsPtr)(lds + (wave * kLoads + j) * 1024), 16, 0, 0);
            src[j] += step;
            at[j] += kSlab;
        }
    }

    // As load, of an across side whose contraction step s is the side's row
    // list[s] / per: the sources are found anew for each slab.
    __device__ void load_listed(char *lds, const void *p, int64_t ld, int64_t row0, int64_t rows,
                                int64_t k_end, const int32_t (&row)[kLoads]) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int q = (wave * kLoads + j) * 64 + lane;
            const int s = q / kPieces, place = q % kPieces;
            const int unit = (place / kUnitPieces) ^ twist(s);
            const int64_t c = row0 + unit * 16 + (place % kUnitPieces) * kElems;
            const int64_t col = c < rows ? c : (rows - 1) / kElems * kElems;
            const char *from = static_cast<const char *>(p) +
                               (row[j] * ld + col) * (int64_t)sizeof(T);
            if (at[j] >= k_end) from = reinterpret_cast<const char *>(&kZeros);
            __builtin_amdgcn_global_load_lds((GlobalPtr)from,
                                             (LdsPtr)(lds + (wave * kLoads + j) * 1024), 16, 0, 0);
            at[j] += kSlab;
        }
    }

    // The rows of the next slab's contraction steps (0 past k_end).
    __device__ void rows_of(const int32_t *list, int per, int64_t k_end, int ahead,
                            int32_t (&row)[kLoads]) const {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int64_t s = at[j] + (int64_t)ahead * kSlab;
            row[j] = s < k_end ? list[s] / per : 0;
        }
    }

    // Fragment of rows r0 .. r0 + 15 and half h (64 bytes of contraction) of a slab.
    static __device__ i4 fragment(const char *lds, int r0, int h) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
        if (!ACROSS) {
            const int r = r0 + i;
            return *reinterpret_cast<const i4 *>(lds + r * 128 + (((h * 4 + g) ^ (r & 7)) << 4));
        }
        constexpr int kRow = ROWS * sizeof(T);
        if (sizeof(T) == 2) {
            s4 v[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int s = 32 * h + 8 * g + 4 * e + (i >> 2);
                const char *from = lds + s * kRow + (((r0 >> 4) ^ twist(s)) << 5) + (i & 3) * 8;
                v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4)from);
            }
            return __builtin_bit_cast(i4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        i4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int s = 16 * h + 4 * g + e;
            v[e] = *reinterpret_cast<const int *>(lds + s * kRow + (((r0 >> 4) ^ twist(s)) << 6) +
                                                  i * 4);
        }
        return v;
    }
};

// --------------------------------------------------------------- the tile
// Which tile a workgroup takes.  Workgroup b runs on XCD b % 8: an XCD takes a
// contiguous range of the tiles, and the tiles are counted in bands of
// kBand rows of tiles, column by column, so that the 32 workgroups that an XCD
// runs at a time read few rows and columns through its L2.
constexpr int kXcds = 8, kBand = 8;

__device__ inline int64_t xcd_tile(int64_t b, int64_t tiles) {
    const int64_t x = b % kXcds, i = b / kXcds, q = tiles / kXcds, r = tiles % kXcds;
    return x * q + (x < r ? x : r) + i;
}

__device__ inline void band_tile(int64_t t, int64_t tm, int64_t tn, int64_t *m, int64_t *n) {
    const int64_t band = t / (kBand * tn), first = band * kBand;
    const int64_t high = tm - first < kBand ? tm - first : kBand;
    const int64_t in = t - band * kBand * tn;
    *m = first + in % high;
    *n = in / high;
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

// Four neighbouring values of a row to and from memory, `left` of them there.
template <typename T>
__device__ inline f4 read4(const T *p, int left, bool vec) {
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if (vec && left >= 4) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        const t4 q = *reinterpret_cast<const t4 *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)q[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) v[e] = (float)p[e];
    }
    return v;
}
template <typename T>
__device__ inline void write4(T *p, f4 v, int left, bool vec) {
    if (vec && left >= 4) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        t4 q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = (T)v[e];
        *reinterpret_cast<t4 *>(p) = q;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (T)v[e];
    }
}

// What happens to four sums of output row `row`, columns `col` .. of batch
// `batch`, before they are rounded and stored.
template <typename T, int MODE>
__device__ inline void epilogue(const ProductArgs &a, int64_t row, int64_t col, int batch, f4 v) {
    const int left = (int)(a.n - col < 4 ? a.n - col : 4);
    const int64_t at = ((MODE == kWeight ? batch * a.m : 0) + row) * a.n + col;
    if (MODE == kForward) {
        if (a.bias)
            v += read4(static_cast<const T *>(a.bias) + batch * a.n + col, left, a.vec & kVecBias);
        if (a.z) write4(static_cast<T *>(a.z) + at, v, left, a.vec & kVecOut);
        if (a.activation != kActNone) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = activate(v[e], a.activation);
        }
        if (a.residual)
            v += read4(static_cast<const T *>(a.residual) + row * a.ldr + col, left,
                       a.vec & kVecResidual);
    }
    if (MODE == kInput && a.slope) {
        const f4 z = read4(static_cast<const T *>(a.slope) + at, left, a.vec & kVecSlope);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= activation_slope(z[e], a.activation);
    }
    write4(static_cast<T *>(a.y) + at, v, left, a.vec & kVecOut);
}

template <typename T, int MODE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64, TM == 256 ? 2 : 1) void product_kernel(ProductArgs a) {
    constexpr bool kAcrossA = MODE == kWeight, kAcrossB = MODE != kForward;
    using SideA = Side<T, kAcrossA, TM, WM * WN>;
    using SideB = Side<T, kAcrossB, TN, WM * WN>;
    constexpr int FM = TM / WM / 16, FN = TN / WN / 16;  // fragments of a wave's tile
    constexpr int kSlab = SideA::kSlab;
    constexpr int kBytes = (TM + TN) * 128;              // of a slab
    extern __shared__ __align__(16) char lds[];

    const int64_t tn = (a.n + TN - 1) / TN;
    int64_t row0, row_end, col0, k0 = 0, k_end = a.k;
    int batch = 0;
    if (MODE == kWeight) {
        const int64_t tm = (a.m + TM - 1) / TM;
        int64_t t = xcd_tile(blockIdx.x, gridDim.x), m, n;
        batch = (int)(t / (tm * tn));
        band_tile(t - batch * tm * tn, tm, tn, &m, &n);
        row0 = m * TM, col0 = n * TN, row_end = a.m;
        if (a.offsets) k0 = a.offsets[batch], k_end = a.offsets[batch + 1];
    } else {
        const int64_t tm = gridDim.x / tn;
        int64_t m, n;
        band_tile(xcd_tile(blockIdx.x, gridDim.x), tm, tn, &m, &n);
        col0 = n * TN;
        if (a.offsets) {
            batch = expert_of(a.offsets, a.experts, TM, m);
            const int64_t first = a.offsets[batch];
            row0 = first + (m - (first / TM + batch)) * TM;
            row_end = a.offsets[batch + 1];
            if (row0 >= row_end) return;
        } else {
            row0 = m * TM, row_end = a.m;
        }
    }
    // this workgroup's part of the contraction
    if (a.splits > 1) {
        const int64_t part = ((k_end - k0 + a.splits - 1) / a.splits + kSlab - 1) / kSlab * kSlab;
        const int64_t from = k0 + part * blockIdx.y;
        k_end = from + part < k_end ? from + part : k_end;
        k0 = from < k_end ? from : k_end;
    }
    const T *pa = static_cast<const T *>(a.a), *pb = static_cast<const T *>(a.b);
    if (MODE != kWeight) pb += batch * a.batch_b;
    const bool listed = MODE == kWeight && a.list;  // side B's rows by the list

    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);

    f4 acc[FM][FN];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y) acc[x][y] = f4{0.f, 0.f, 0.f, 0.f};
    // gradient of the bias: the sums of side A over the contraction, as a product
    // with ones on the workgroups and waves of the first columns
    const bool sums = MODE == kWeight && a.bias_grad && col0 == 0 && wn == 0;
    f4 sum[MODE == kWeight ? FM : 1];
#pragma unroll
    for (int x = 0; x < (MODE == kWeight ? FM : 1); ++x) sum[x] = f4{0.f, 0.f, 0.f, 0.f};
    i4 ones;
    {
        const int one = sizeof(T) == 4 ? 0x3f800000
                        : __is_same(T, __bf16) ? 0x3f803f80 : 0x3c003c00;
        ones = i4{one, one, one, one};
    }

    const int64_t slabs = (k_end - k0 + kSlab - 1) / kSlab;
    if (slabs > 0) {
        SideA sa;
        SideB sb;
        sa.begin(pa, a.lda, row0, row_end, k0, MODE == kWeight ? nullptr : a.list, a.per);
        sb.begin(pb, a.ldb, col0, a.n, k0, nullptr, 1);
        int32_t row[SideB::kLoads];
        if (MODE == kWeight && listed) sb.rows_of(a.list, a.per, k_end, 0, row);
        const auto load = [&](int64_t s) {
            char *to = lds + (s & 1) * kBytes;
            const bool whole = k0 + (s + 1) * kSlab <= k_end;
            sa.load(to, k_end, whole);
            if (MODE == kWeight && listed) {
                sb.load_listed(to + TM * 128, pb, a.ldb, col0, a.n, k_end, row);
                sb.rows_of(a.list, a.per, k_end, 0, row);
            } else {
                sb.load(to + TM * 128, k_end, whole);
            }
        };
        load(0);
        for (int64_t s = 0; s < slabs; ++s) {
            __builtin_amdgcn_s_waitcnt(0x0F70);  // this wave's loads of slab s are in LDS
            __syncthreads();                     // and everyone's; slab s - 1 is no longer read
            if (s + 1 < slabs) load(s + 1);
            const char *la = lds + (s & 1) * kBytes, *lb = la + TM * 128;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                i4 fa[FM], fb[FN];
#pragma unroll
                for (int x = 0; x < FM; ++x) fa[x] = SideA::fragment(la, wm + 16 * x, h);
#pragma unroll
                for (int y = 0; y < FN; ++y) fb[y] = SideB::fragment(lb, wn + 16 * y, h);
#pragma unroll
                for (int x = 0; x < FM; ++x)
#pragma unroll
                    for (int y = 0; y < FN; ++y)
                        acc[x][y] = multiply<T>(fb[y], fa[x], acc[x][y]);
                if (MODE == kWeight && sums) {
#pragma unroll
                    for (int x = 0; x < FM; ++x) sum[x] = multiply<T>(ones, fa[x], sum[x]);
                }
            }
        }
    }

#pragma unroll
    for (int x = 0; x < FM; ++x) {
        const int64_t row = row0 + wm + 16 * x + i;
        if (row >= row_end) continue;
#pragma unroll
        for (int y = 0; y < FN; ++y) {
            const int64_t col = col0 + wn + 16 * y + 4 * g;
            if (col >= a.n) continue;
            if (a.splits > 1) {  // columns are padded to whole tiles
                const int64_t ld = tn * TN;
                const int64_t r = MODE == kWeight ? (int64_t)batch * a.m + row : row;
                *reinterpret_cast<f4 *>(a.partial + (blockIdx.y * a.partial_rows + r) * ld + col) =
                    acc[x][y];
            } else {
                epilogue<T, MODE>(a, row, col, batch, acc[x][y]);
            }
        }
        if (MODE == kWeight && sums && g == 0) {
            const int64_t r = (int64_t)batch * a.m + row;
            if (a.splits > 1)
                a.partial[a.splits * a.partial_rows * tn * TN + blockIdx.y * a.partial_rows + r] =
                    sum[x][0];
            else
                static_cast<T *>(a.bias_grad)[r] = (T)sum[x][0];
        }
    }
}

// Joins the parts of a split contraction, in order, and ends the product: four
// columns a thread.  ld: columns of the partial sums.
template <typename T, int MODE>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a, int64_t ld) {
    const int64_t quads = (a.n + 3) / 4;
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = q / quads, col = q % quads * 4;
    if (r < a.partial_rows) {
        int batch = 0;
        int64_t row = r;
        bool there = true;
        if (MODE == kWeight) {
            batch = (int)(r / a.m);
            row = r % a.m;
        } else if (a.offsets) {
            there = r < a.offsets[a.experts];
            for (int hi = a.experts; hi - batch > 1;) {  // the expert whose rows hold r
                const int mid = (batch + hi) / 2;
                if (a.offsets[mid] <= r) batch = mid;
                else hi = mid;
            }
        }
        if (there) {
            f4 v = {0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < a.splits; ++s)
                v += *reinterpret_cast<const f4 *>(a.partial + (s * a.partial_rows + r) * ld + col);
            epilogue<T, MODE>(a, row, col, batch, v);
        }
    }
    if (MODE == kWeight && a.bias_grad && q < a.partial_rows) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s)
            v += a.partial[a.splits * a.partial_rows * ld + s * a.partial_rows + q];
        static_cast<T *>(a.bias_grad)[q] = (T)v;
    }
}

// Forward product of few rows (16 R at a time): bound by one read of w.  A
// workgroup takes 16 columns of C, its waves take the contraction's slabs in
// turn, straight from memory into the fragments (no LDS: w is used once, x
// comes from the caches), several slabs in flight, and join their sums through
// LDS in order.  VEC: pieces are 16-byte aligned; otherwise they are read
// element by element.
template <typename T, bool VEC>
__device__ inline i4 piece(const T *row, int64_t k, int64_t k_end) {
    constexpr int kElems = 16 / sizeof(T);
    if (VEC) {
        const void *from = k < k_end ? static_cast<const void *>(row + k) : &kZeros;
        return *static_cast<const i4 *>(from);
    }
    typedef T te __attribute__((ext_vector_type(kElems)));
    te v;
#pragma unroll
    for (int e = 0; e < kElems; ++e) v[e] = k + e < k_end ? row[k + e] : (T)0.f;
    return __builtin_bit_cast(i4, v);
}

template <typename T, int R, int WAVES, bool VEC>
__global__ __launch_bounds__(WAVES * 64) void rows_kernel(ProductArgs a, int by_row) {
    constexpr int kElems = 16 / sizeof(T), kSlab = 128 / sizeof(T), kAhead = R == 1 ? 4 : 2;
    __shared__ f4 part[WAVES][R][64];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
    int batch = 0;
    int64_t row0 = (int64_t)blockIdx.y * 16 * R, row_end = a.m;
    if (a.offsets) {
        const int64_t t = blockIdx.y;
        batch = expert_of(a.offsets, a.experts, by_row ? 0 : 16 * R, t);
        const int64_t first = a.offsets[batch];
        row_end = a.offsets[batch + 1];
        row0 = by_row ? t : first + (t - (first / (16 * R) + batch)) * (16 * R);
        if (row0 >= row_end || (by_row && (t - first) % (16 * R) != 0)) return;
    }
    const int64_t col0 = (int64_t)blockIdx.x * 16;
    const T *wr = static_cast<const T *>(a.b) + batch * a.batch_b +
                  (col0 + i < a.n ? col0 + i : a.n - 1) * a.ldb;
    const T *xr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        int64_t row = row0 + 16 * r + i < row_end ? row0 + 16 * r + i : row_end - 1;
        if (a.list) row = a.list[row] / a.per;
        xr[r] = static_cast<const T *>(a.a) + row * a.lda;
    }
    f4 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = f4{0.f, 0.f, 0.f, 0.f};
    for (int64_t k = (int64_t)wave * kSlab; k < a.k; k += (int64_t)kAhead * WAVES * kSlab) {
        i4 fw[kAhead][2], fx[kAhead][2][R];
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = k + (int64_t)s * WAVES * kSlab + (h * 4 + g) * kElems;
                fw[s][h] = piece<T, VEC>(wr, c, a.k);
#pragma unroll
                for (int r = 0; r < R; ++r) fx[s][h][r] = piece<T, VEC>(xr[r], c, a.k);
            }
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < R; ++r)
                    acc[r] = multiply<T>(fw[s][h], fx[s][h][r], acc[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) part[wave][r][lane] = acc[r];
    __syncthreads();
    for (int r = wave; r < R; r += WAVES) {
        f4 v = part[0][r][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += part[w][r][lane];
        const int64_t row = row0 + 16 * r + i, col = col0 + 4 * g;
        if (row < row_end && col < a.n) epilogue<T, kForward>(a, row, col, batch, v);
    }
}

template <typename T, int MODE, int TM, int TN, int WM, int WN>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t stream) {
    const int64_t tn = (a.n + TN - 1) / TN;
    const int64_t tm = MODE == kWeight ? (a.m + TM - 1) / TM * (a.offsets ? a.experts : 1)
                       : a.offsets     ? a.m / TM + a.experts
                                       : (a.m + TM - 1) / TM;
    if (tm * tn > INT32_MAX) return hipErrorInvalidValue;
    constexpr int kLds = 2 * (TM + TN) * 128;
    const auto kernel = product_kernel<T, MODE, TM, TN, WM, WN>;
    if (kLds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)(tm * tn), a.splits), WM * WN * 64, kLds, stream>>>(a);
    if (a.splits > 1) {
        const int64_t quads = std::max(a.partial_rows * ((a.n + 3) / 4), a.partial_rows);
        if ((quads + 255) / 256 > INT32_MAX) return hipErrorInvalidValue;
        join_kernel<T, MODE><<<(unsigned)((quads + 255) / 256), 256, 0, stream>>>(a, tn * TN);
    }
    return hipGetLastError();
}

template <typename T, int MODE>
hipError_t launch_mode(const ProductArgs &a, const ProductPlan &p, hipStream_t stream) {
    switch (p.tile) {
        case 256: return launch_tiles<T, MODE, 256, 256, 2, 4>(a, stream);
        case 128: return launch_tiles<T, MODE, 128, 128, 2, 2>(a, stream);
        default: return launch_tiles<T, MODE, 64, 64, 2, 2>(a, stream);
    }
}

template <typename T, int R, int WAVES>
hipError_t launch_rows(const ProductArgs &a, bool aligned, hipStream_t stream) {
    const int64_t tiles = a.offsets ? a.m / (16 * R) + a.experts : (a.m + 16 * R - 1) / (16 * R);
    const int by_row = a.offsets && a.m < tiles;
    const int64_t high = by_row ? a.m : tiles;
    const int64_t wide = (a.n + 15) / 16;
    if (high > 65535 || wide > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wide, (unsigned)high);
    if (aligned) rows_kernel<T, R, WAVES, true><<<grid, WAVES * 64, 0, stream>>>(a, by_row);
    else rows_kernel<T, R, WAVES, false><<<grid, WAVES * 64, 0, stream>>>(a, by_row);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_product(ProductArgs a, const ProductPlan &p, hipStream_t stream) {
    a.splits = p.splits;
    if (p.tile <= 64 && p.waves) {
        const bool al = p.aligned;
        if (p.tile == 16) return p.waves == 4 ? launch_rows<T, 1, 4>(a, al, stream)
                                              : launch_rows<T, 1, 16>(a, al, stream);
        return p.waves == 4 ? launch_rows<T, 4, 4>(a, al, stream)
                            : launch_rows<T, 4, 16>(a, al, stream);
    }
    switch (a.mode) {
        case kForward: return launch_mode<T, kForward>(a, p, stream);
        case kInput: return launch_mode<T, kInput>(a, p, stream);
        default: return launch_mode<T, kWeight>(a, p, stream);
    }
}

}  // namespace
}  // namespace som
