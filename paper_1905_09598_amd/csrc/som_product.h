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
// Rows beyond C are read from its last row, columns from its first, and not
// stored; the contraction is filled up from 16 bytes of zeros.
#pragma once

#include "som_local_internal.h"

#include <algorithm>
#include <type_traits>

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
// ROWS rows (or columns) of a tile, loaded by WAVES waves.  A lane's source is a
// 32-bit offset from a base that all lanes share and that moves from slab to
// slab (the launcher sees to it that the offsets fit).
//
// DMA: pieces go straight to LDS; they have to be whole and 16-byte aligned (the
// columns of an across side a multiple of a piece, so that none crosses a row's
// end).  Without, rows may begin anywhere and pieces go through registers.  An
// across side's pieces that cross a row's end hold columns that are not stored:
// what follows the row is read with them (`easy`), except where nothing need
// follow, in the last slab, in rows named by a list, and in rows shorter than a
// piece; there they are read element by element.
template <typename T, bool ACROSS, bool DMA, int ROWS, int WAVES>
struct Side {
    static constexpr int kElems = 16 / sizeof(T);           // elements of a 16-byte piece
    static constexpr int kSlab = 128 / sizeof(T);           // contraction of a slab
    static constexpr int kLoads = ROWS / 8 / WAVES;         // 1 KB each, per wave
    static constexpr int kPieces = ROWS / kElems;           // across: pieces of a step
    static constexpr int kUnits = ROWS / 16;                // across: units of 16 columns
    static constexpr int kUnitPieces = 16 / kElems;
    static_assert(kLoads * WAVES * 8 == ROWS, "whole loads");

    const char *base;
    uint32_t off[kLoads];
    int64_t step;             // bytes from slab to slab
    i4 held[DMA ? 1 : kLoads];
    bool easy;                // tells all lanes alike

    // What the units of contraction step s are exchanged with.
    static __device__ int twist(int s) {
        const int f = sizeof(T) == 2 ? (s & 3) | ((s >> 3) & 1) << 2 : (s >> 2) & 3;
        return f & (kUnits - 1);
    }
    // The 16-byte place in the LDS slab that load j of this lane fills.
    static __device__ int place(int j) {
        return ((threadIdx.x >> 6) * kLoads + j) * 64 + (threadIdx.x & 63);
    }
    // Its contraction index within the slab.
    static __device__ int index(int j) {
        const int q = place(j);
        return ACROSS ? q / kPieces : ((q & 7) ^ (q >> 3 & 7)) * kElems;
    }
    // across: the column it holds, another one beyond the matrix.
    static __device__ int64_t column(int j, int64_t col0, int64_t cols) {
        const int q = place(j), s = q / kPieces, at = q % kPieces;
        const int unit = (at / kUnitPieces) ^ twist(s);
        const int64_t c = col0 + unit * 16 + (at % kUnitPieces) * kElems;
        return c < cols ? c : 0;
    }

    // Rows row0 .. of a side of `rows` rows whose element (r, c) is p[r * ld + c]
    // (along), or columns row0 .. of one whose element is p[c * ld + r] (across),
    // from contraction index k0 on; `list`: row r is the side's row list[r] / per.
    __device__ void begin(const T *p, int64_t ld, int64_t row0, int64_t rows, int64_t k0,
                          const int32_t *list, Divider per) {
        base = reinterpret_cast<const char *>(p + (ACROSS ? k0 * ld : k0 + (list ? 0 : row0 * ld)));
        step = ACROSS ? kSlab * ld * (int64_t)sizeof(T) : 128;
        easy = row0 + ROWS <= rows || ld >= kElems;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            if (ACROSS) {
                off[j] = (uint32_t)((index(j) * ld + column(j, row0, rows)) * (int64_t)sizeof(T));
            } else {
                const int r = place(j) >> 3;
                int64_t row = row0 + r < rows ? r : rows - 1 - row0;
                if (list) row = per.quotient(list[row0 + row]);
                off[j] = (uint32_t)((row * ld + index(j)) * (int64_t)sizeof(T));
            }
        }
    }

    // Load the next slab, with DMA into `lds`.  CHECK: `left` contraction indices are
    // left, the rest are zeros.  across: columns col0 .. of `cols`.
    template <bool CHECK>
    __device__ void load(char *lds, int64_t left, int64_t col0, int64_t cols) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        if (!DMA && !CHECK && (!ACROSS || easy)) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                __builtin_memcpy(&held[j], __builtin_assume_aligned(base + off[j], sizeof(T)), 16);
            base += step;
            return;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const char *from = base + off[j];
            if (DMA) {
                if (CHECK && index(j) >= left) from = reinterpret_cast<const char *>(&kZeros);
                __builtin_amdgcn_global_load_lds((GlobalPtr)from,
                                                 (LdsPtr)(lds + (wave * kLoads + j) * 1024), 16, 0,
                                                 0);
            } else {
                int64_t here = kElems;   // elements of the piece that are there
                if (ACROSS) here = cols - column(j, col0, cols);
                if (CHECK && ACROSS && index(j) >= left) here = 0;
                if (CHECK && !ACROSS) here = left - index(j);
                if (here >= kElems) {
                    __builtin_memcpy(&held[j], __builtin_assume_aligned(from, sizeof(T)), 16);
                } else {
                    typedef T Vec __attribute__((ext_vector_type(kElems)));
                    Vec v;
#pragma unroll
                    for (int e = 0; e < kElems; ++e)
                        v[e] = e < here ? reinterpret_cast<const T *>(from)[e] : (T)0.f;
                    held[j] = __builtin_bit_cast(i4, v);
                }
            }
        }
        base += step;
    }
    // Without DMA: what was loaded last, into `lds`.
    __device__ void store(char *lds) const {
#pragma unroll
        for (int j = 0; j < (DMA ? 0 : kLoads); ++j)
            *reinterpret_cast<i4 *>(lds + place(j) * 16) = held[j];
    }

    // An across side whose contraction step s is the matrix's row list[s] / per:
    // the list's entries for the next slab (it points at the slab's first), and the
    // offsets that they give.
    __device__ static void entries(const int32_t *list, int64_t left, int32_t (&row)[kLoads]) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) row[j] = index(j) < left ? list[index(j)] : 0;
    }
    __device__ void follow(const int32_t (&row)[kLoads], Divider per, int64_t ld, int64_t col0,
                           int64_t cols) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            off[j] = (uint32_t)(((int64_t)per.quotient(row[j]) * ld + column(j, col0, cols)) *
                                (int64_t)sizeof(T));
    }
};

// Where a wave's F fragments lie in a side's LDS slab: one offset that depends on
// the lane.  Fragment f's differs from it by a constant (along), or by an
// exclusive or, as the fragments' numbers and the twist are (across); that is done
// anew for every slab, so that it takes an instruction and not a register.
template <typename T, bool ACROSS, int ROWS, int F>
struct Fragments {
    static_assert((F & (F - 1)) == 0, "the first fragment's number is a multiple of F");
    static constexpr int kRow = ROWS * sizeof(T);   // across: bytes of a contraction step
    int at;

    // The wave's fragments begin at row r0 of the tile.
    __device__ void begin(int r0) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
        if (!ACROSS) {
            at = (r0 + i) * 128 + ((g ^ (i & 7)) << 4);
        } else {
            const int s = sizeof(T) == 2 ? 8 * g + (i >> 2) : 4 * g;
            const int unit = r0 / 16 ^ Side<T, true, true, ROWS, ROWS / 8>::twist(s);
            at = s * kRow + unit * 16 * (int)sizeof(T) + (sizeof(T) == 2 ? (i & 3) * 8 : i * 4);
        }
    }
    // Fragment f, half h (64 bytes of contraction) of the slab at lds + slab, a
    // multiple of all that is exchanged.
    __device__ i4 read(const char *lds, int slab, int f, int h) const {
        if (!ACROSS)
            return *reinterpret_cast<const i4 *>(lds + ((slab + at) ^ (h * 64)) + f * 16 * 128);
        const char *from = lds + ((slab + at) ^ (f * 16 * (int)sizeof(T)));
        if (sizeof(T) == 2) {
            s4 v[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (LdsS4)(from + (32 * h + 4 * e) * kRow));
            return __builtin_bit_cast(i4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        i4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = *reinterpret_cast<const int *>(from + (16 * h + e) * kRow);
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

// The activation of N values.
template <int N>
__device__ inline void activate_all(float (&v)[N], int32_t kind) {
    if (kind == kActRelu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], kActRelu);
    } else if (kind == kActGelu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], kActGelu);
    } else if (kind == kActSilu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], kActSilu);
    }
}
// The activation of N values in place of them, and its slopes.
template <int N>
__device__ inline void slopes_all(float (&v)[N], float (&slope)[N], int32_t kind) {
    if (kind == kActRelu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], kActRelu, &slope[e]);
    } else if (kind == kActGelu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], kActGelu, &slope[e]);
    } else if (kind == kActSilu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], kActSilu, &slope[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) slope[e] = 1.f;
    }
}

// Waits until at most COUNT of this wave's loads are under way.
template <int COUNT>
__device__ inline void wait_loads() {
    __builtin_amdgcn_s_waitcnt((COUNT & 15) | (COUNT >> 4 & 3) << 14 | 0x0F70);
}

template <int V>
using Int = std::integral_constant<int, V>;

// What happens to N sums of output row `row`, columns `col` .. of batch `batch`,
// before they are rounded and stored: in two steps, so that the reads of several
// rows can be under way together.
template <typename T, int MODE, int N>
struct Epilogue {
    const ProductArgs &a;
    int64_t col;
    int batch, left;
    float bias[N];
    static constexpr bool kImage = MODE == kGate && sizeof(T) == 2;
    // Beside a row's sums: its residual (forward) or the argument of its activation
    // (gate), and the weight of its slot.
    struct Row {
        Piece<T, N> piece;
        float gate;
    };
    __device__ Epilogue(const ProductArgs &args, int64_t c, int b) : a(args), col(c), batch(b) {
        left = (int)(a.n - col < N ? a.n - col : N);
        Piece<T, N> p;
        const bool there = MODE == kForward && a.bias && left > 0;
        if (there) p.read(static_cast<const T *>(a.bias) + batch * a.n + col, left);
#pragma unroll
        for (int e = 0; e < N; ++e) bias[e] = there ? (float)p.v[e] : 0.f;
    }
    // The part of a weight that an activation is kept with.
    __device__ static float kept_part(float gate) {
        return std::is_same<T, _Float16>::value ? gate_kept(gate) : gate;
    }
    __device__ static void read(const ProductArgs &a, int64_t row, int64_t col, Row &r) {
        const int left = (int)(a.n - col < N ? a.n - col : N);
        if (MODE == kForward) {
            if (a.residual)
                r.piece.read(static_cast<const T *>(a.residual) + row * a.ldr + col, left);
            if (a.scaled) r.gate = kept_part(a.gates ? a.gates[a.slots[row]] : 1.f);
        }
        if (MODE == kGate) {
            const int slot = a.slots[row];
            r.gate = a.gates ? a.gates[slot] : 1.f;
            r.piece.read(static_cast<const T *>(a.argument) +
                             (a.argument_listed ? (int64_t)a.per.quotient(slot) : row) * a.ld_argument + col,
                         left);
        }
    }
    __device__ void store(void *to, int64_t at, const float (&v)[N]) const {
        Piece<T, N> out;
#pragma unroll
        for (int e = 0; e < N; ++e) out.v[e] = (T)v[e];
        out.write(static_cast<T *>(to) + at, left);
    }
    // z as a gradient takes it.  A finite sum stays finite (slopes of infinities are not
    // numbers; at the type's largest magnitude they are 0 and 1), and for relu, whose slope
    // goes by the sign, what is positive stays positive where the type would round it to 0.
    __device__ void keep(int64_t at, const float (&v)[N]) const {
        if (a.activation == kActNone || sizeof(T) == 4) return store(a.z, at, v);
        constexpr bool half = std::is_same<T, _Float16>::value;
        constexpr float most = half ? 65504.f : 0x1.fep127f, least = half ? 0x1p-24f : 0x1p-133f;
        float u[N], top = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = v[e], top = fmaxf(top, fabsf(v[e]));
        if (top > most) {   // seldom
#pragma unroll
            for (int e = 0; e < N; ++e)
                u[e] = fabsf(v[e]) < INFINITY ? __builtin_amdgcn_fmed3f(v[e], -most, most) : v[e];
        }
        if (a.activation == kActRelu) {
#pragma unroll
            for (int e = 0; e < N; ++e) u[e] = v[e] > 0.f ? fmaxf(u[e], least) : u[e];
        }
        store(a.z, at, u);
    }
    // gate: returns the sum of the products with the activation; image: a.image's.
    __device__ float write(int64_t row, const Row &r, const Piece<T, N> &image, float (&v)[N]) const {
        const int64_t at = ((MODE == kWeight ? batch * a.m : 0) + row) * a.n + col;
        float dot = 0.f;
        if (MODE == kForward) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += bias[e];
            if (a.z) keep(at, v);
            activate_all(v, a.activation);
            if (a.scaled) {
                float u[N];
#pragma unroll
                for (int e = 0; e < N; ++e) u[e] = r.gate * v[e];
                store(a.scaled, at, u);
            }
            if (a.residual) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] += (float)r.piece.v[e];
            }
        }
        if (MODE == kGate) {
            float h[N], slope[N];
#pragma unroll
            for (int e = 0; e < N; ++e) h[e] = (float)r.piece.v[e];
            slopes_all(h, slope, a.activation);
            if (kImage && a.image) {
                // image / gate is the same activation, rounded by itself (unless it was
                // too small or too large for its type): the mean of the two is off by less.
                // Gates whose reciprocal is no normal number (a softmax has weights down to
                // 0) take no part.
                const float gate = kept_part(r.gate), by = __builtin_amdgcn_rcpf(gate);
                const bool usable = fabsf(gate) >= 0x1p-126f && fabsf(gate) <= 0x1p126f;
                const float least =
                    !usable ? INFINITY : std::is_same<T, __bf16>::value ? 0x1p-126f : 0x1p-14f;
                constexpr float most = std::is_same<T, __bf16>::value ? 0x1p127f : 65504.f;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float u = (float)image.v[e];
                    const bool fine = fabsf(u) >= least && fabsf(u) <= most;
                    h[e] = fine ? 0.5f * (h[e] + u * by) : h[e];
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                dot = e < left ? fmaf(v[e], h[e], dot) : dot;
                v[e] *= r.gate * slope[e];
            }
        }
        if ((MODE == kForward || MODE == kInput || MODE == kGate) && a.wide) {
            Piece<float, N> out;
#pragma unroll
            for (int e = 0; e < N; ++e) out.v[e] = v[e];
            out.write(static_cast<float *>(a.y) + at, left);
        } else {
            store(a.y, at, v);
        }
        return dot;
    }
};

// A workgroup's tile: WM x WN waves of (TM / WM) x (TN / WN).  Per slab, with the
// fragments of its first half in registers:
//   read the second half's fragments; multiply the first
//   wait: the next slab has landed, and nobody reads this one any more
//   load the slab after the next in its place; read the next slab's first half;
//   multiply the second half
// so that the matrix cores always have fragments in hand, and a load has a slab's
// time to arrive.  8192 x 2048 x 8192 in bf16 takes 229 us in tiles of 256 (1200 TFLOP/s),
// 256 in 128s and 360 in 64s, 282 with bias, gelu and a residual (one workgroup holds a
// compute unit, and nothing else runs beside its epilogue); 16,001 x 2048 x 2048 in fp16
// 124, 138 and 191 us: the larger the tile, the fewer reads a product.  The first, with
// its epilogue, holds the matrix cores for 43 % of its cycles and LDS for 18 %, without a
// bank conflict, at 2.05 GHz, and fetches 269 MB of the 201 it needs: bound by what the
// slabs and the epilogue wait for.  Small tiles fill the chip where there are few
// (plan_product).
template <typename T, int MODE, int LIST, bool DMA, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(ProductArgs a) {
    constexpr bool kAcrossA = MODE == kWeight, kAcrossB = MODE != kForward;
    constexpr bool LISTED = LIST != 0;
    using SideA = Side<T, kAcrossA, DMA, TM, WM * WN>;
    using SideB = Side<T, kAcrossB, DMA, TN, WM * WN>;
    constexpr int kTileM = TM / WM, kTileN = TN / WN;    // of a wave
    constexpr int FM = kTileM / 16, FN = kTileN / 16;    // its fragments
    constexpr int kSlab = SideA::kSlab;
    constexpr int kBytes = (TM + TN) * 128;              // of a slab
    extern __shared__ __align__(16) char lds[];

    const int64_t tn = (a.n + TN - 1) / TN;
    int64_t row0, row_end, col0, k0 = 0, k_end = a.k;
    int batch = 0;
    if (MODE == kWeight) {
        // expert by expert, the largest first, each over all XCDs: a tile's time is
        // its expert's rows
        const unsigned tm = (unsigned)((a.m + TM - 1) / TM), tiles = tm * (unsigned)tn;
        batch = (int)(blockIdx.x / tiles);
        int64_t m, n;
        band_tile(xcd_tile(blockIdx.x - batch * tiles, tiles), tm, tn, &m, &n);
        row0 = m * TM, col0 = n * TN, row_end = a.m;
        if (a.offsets) {
            batch = expert_of_rank(a.offsets, a.experts, batch);
            k0 = a.offsets[batch], k_end = a.offsets[batch + 1];
        }
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

    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN * kTileM, wn = wave % WN * kTileN;

    f4 acc[FM][FN];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y) acc[x][y] = f4{0.f, 0.f, 0.f, 0.f};
    // The result's rows as they leave: N columns a lane, kPass rows of the wave at a
    // time; what lies beside them in memory is read kGroup passes ahead.
    constexpr int N = 16 / sizeof(T), kQuads = kTileN / 4;
    constexpr int kFits = 2 * kBytes / (WM * WN * kTileN * 4);   // rows of a wave's part
    constexpr int kMost = kFits >= 64 ? 64 : kFits >= 32 ? 32 : 16;
    constexpr int kRowsAt = kTileM < kMost ? kTileM : kMost;
    constexpr int kLanes = kTileN / N, kPass = 64 / kLanes;
    constexpr int kGroup = kRowsAt / kPass < 4 ? kRowsAt / kPass : 4;
    static_assert(WM * WN * kRowsAt * kTileN * 4 <= 2 * kBytes, "fits in the slabs' LDS");
    using Row = typename Epilogue<T, MODE, N>::Row;
    f4 *mine = reinterpret_cast<f4 *>(lds) + wave * (kRowsAt * kQuads);
    const int64_t col = col0 + wn + lane % kLanes * N;
    Row extra[kGroup];
    const auto beside = [&](int r0, Row (&to)[kGroup]) {
        if (a.splits > 1 || col >= a.n) return;
#pragma unroll
        for (int q = 0; q < kGroup; ++q) {
            const int r = r0 + q * kPass + lane / kLanes;
            if (r < kTileM && row0 + wm + r < row_end)
                Epilogue<T, MODE, N>::read(a, row0 + wm + r, col, to[q]);
        }
    };

    const int64_t slabs = (k_end - k0 + kSlab - 1) / kSlab;
    if (slabs == 0) beside(0, extra);
    if (slabs > 0) {
        SideA sa;
        SideB sb;
        Fragments<T, kAcrossA, TM, FM> ra;
        Fragments<T, kAcrossB, TN, FN> rb;
        sa.begin(pa, a.lda, row0, row_end, LIST == 2 ? 0 : k0, MODE == kWeight ? nullptr : a.list,
                 a.per);
        sb.begin(pb, a.ldb, col0, a.n, LIST == 1 ? 0 : k0, nullptr, a.per);
        ra.begin(wm);
        rb.begin(wn);
        int32_t entry[LIST == 2 ? SideA::kLoads : SideB::kLoads];
        const auto entries = [&](int64_t s) {
            if constexpr (LIST == 1) SideB::entries(a.list + k0 + s * kSlab, k_end - k0 - s * kSlab, entry);
            if constexpr (LIST == 2) SideA::entries(a.list + k0 + s * kSlab, k_end - k0 - s * kSlab, entry);
        };
        if (LIST == 1) sb.step = 0, sb.easy = col0 + TN <= a.n;
        if (LIST == 2) sa.step = 0, sa.easy = row0 + TM <= row_end;
        entries(0);
        // the offsets of the slab that is loaded next, and the list beyond it
        const auto follow = [&](int64_t s) {
            if constexpr (LIST == 1) sb.follow(entry, a.per, a.ldb, col0, a.n);
            if constexpr (LIST == 2) sa.follow(entry, a.per, a.lda, row0, row_end);
            entries(s + 1);
        };
        const auto load = [&](auto check, int64_t s) {
            char *to = lds + (s & 1) * kBytes;
            const int64_t left = k_end - k0 - s * kSlab;
            sa.template load<decltype(check)::value>(to, left, row0, row_end);
            sb.template load<decltype(check)::value>(to + TM * 128, left, col0, a.n);
        };
        const auto store = [&](int64_t s) {
            sa.store(lds + (s & 1) * kBytes);
            sb.store(lds + (s & 1) * kBytes + TM * 128);
        };
        i4 fa[2][FM], fb[2][FN];
        const auto read = [&](int64_t s, auto half) {
            constexpr int h = decltype(half)::value;
            const int la = (int)(s & 1) * kBytes, lb = la + TM * 128;
#pragma unroll
            for (int y = 0; y < FN; ++y) fb[h][y] = rb.read(lds, lb, y, h);
#pragma unroll
            for (int x = 0; x < FM; ++x) fa[h][x] = ra.read(lds, la, x, h);
        };
        const auto times = [&](auto half) {
            constexpr int h = decltype(half)::value;
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; ++y)
                    acc[x][y] = multiply<T>(fb[h][y], fa[h][x], acc[x][y]);
        };
        // slab s; loading slab s + 2 (2: of a whole slab, 1: perhaps the last, in part),
        // or only going on to slab s + 1 (0), or not even that (-1)
        const auto slab = [&](auto what, int64_t s) {
            constexpr int k = decltype(what)::value;
            if (k > 0) follow(s + 2);
            read(s, Int<1>());
            times(Int<0>());
            __builtin_amdgcn_sched_barrier(0);   // the products come before the waits
            if (k < 0) {
                beside(0, extra);
                times(Int<1>());
                return;
            }
            if (DMA) wait_loads<0>();            // the next slab has landed
            else store(s + 1);
            __syncthreads();                     // for everyone; this one is no longer read
            if (k == 2) load(Int<0>(), s + 2);
            if (k == 1) load(Int<1>(), s + 2);
            read(s + 1, Int<0>());
            times(Int<1>());
            __builtin_amdgcn_sched_barrier(0);
        };
        follow(0);
        load(Int<1>(), 0);
        store(0);
        if (slabs > 1) {
            follow(1);
            load(Int<1>(), 1);
        }
        // all but the second slab's loads have landed
        if (DMA && slabs > 1 && !LISTED) wait_loads<SideA::kLoads + SideB::kLoads>();
        else if (DMA) wait_loads<0>();
        __syncthreads();
        read(0, Int<0>());
        int64_t s = 0;
        for (; s + 3 < slabs; ++s) slab(Int<2>(), s);
        if (s + 2 < slabs) slab(Int<1>(), s++);
        if (s + 1 < slabs) slab(Int<0>(), s++);
        slab(Int<-1>(), s);
    }

    // Through LDS, so that a lane holds 16 bytes of a row of the result: the
    // waves' own parts, up to 64 rows at a time, quads of columns exchanged by row so
    // that all banks are met.
    __syncthreads();
    const Epilogue<T, MODE, N> end(a, col < a.n ? col : 0, batch);
#pragma unroll
    for (int x0 = 0; x0 < FM; x0 += kRowsAt / 16) {
#pragma unroll
        for (int x = 0; x < kRowsAt / 16; ++x)
#pragma unroll
            for (int y = 0; y < FN; ++y)
                mine[(16 * x + i) * kQuads + ((4 * y + g) ^ (i & (kQuads - 1)))] = acc[x0 + x][y];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
        for (int p = 0; p < kRowsAt / kPass; p += kGroup) {
            // what lies beside the next rows is read while these are worked on
            Row next[kGroup];
            beside(16 * x0 + (p + kGroup) * kPass, next);
            Piece<T, N> image[kGroup];
            if (Epilogue<T, MODE, N>::kImage && a.image && col < a.n) {
#pragma unroll
                for (int q = 0; q < kGroup; ++q) {
                    const int64_t row = row0 + wm + 16 * x0 + (p + q) * kPass + lane / kLanes;
                    if (row < row_end)
                        image[q].read(static_cast<const T *>(a.image) + row * a.n + col, end.left);
                }
            }
#pragma unroll
            for (int q = 0; q < kGroup; ++q) {
                const int r = (p + q) * kPass + lane / kLanes;
                const int64_t row = row0 + wm + 16 * x0 + r;
                float v[N];
#pragma unroll
                for (int e = 0; e < N / 4; ++e) {
                    const f4 u = mine[r * kQuads + ((lane % kLanes * (N / 4) + e) ^
                                                    (r & 15 & (kQuads - 1)))];
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[4 * e + c] = u[c];
                }
                const bool there = row < row_end && col < a.n;
                float dot = 0.f;
                if (there && a.splits > 1) {  // columns are padded to whole tiles
                    const int64_t at = MODE == kWeight ? (int64_t)batch * a.m + row : row;
                    f4 *to = reinterpret_cast<f4 *>(
                        a.partial + (blockIdx.y * a.partial_rows + at) * (tn * TN) + col);
#pragma unroll
                    for (int e = 0; e < N / 4; ++e)
                        to[e] = f4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
                } else if (there) {
                    dot = end.write(row, extra[q], image[q], v);
                }
                if (MODE == kGate) {   // the lanes of a row together
#pragma unroll
                    for (int o = 1; o < kLanes; o <<= 1) dot += __shfl_xor(dot, o);
                    if (there && lane % kLanes == 0)
                        a.dots[row * a.dot_cols + (col0 + wn) / kTileN] = dot;
                }
            }
#pragma unroll
            for (int q = 0; q < kGroup; ++q) extra[q] = next[q];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
            float u[4] = {v[0], v[1], v[2], v[3]};
            const Epilogue<T, MODE, 4> end(a, col, batch);
            typename Epilogue<T, MODE, 4>::Row extra;
            end.read(a, row, col, extra);
            end.write(row, extra, {}, u);
        }
    }
}

// Forward product of few rows, 16 at a time: bound by one read of w.  A workgroup
// takes 16 columns of C, its waves take the contraction's slabs in turn, straight
// from memory into the fragments (no LDS: w is used once, x comes from the
// caches), four slabs in flight, and join their sums through LDS in order.
// Measured here and in tiles (us): one row of 2048 by 10,000 in bf16 10.4 (3.9 TB/s) and
// 13.8; sixteen rows, one fragment, 14.0 and 13.7, of 2048 by 1024 6.1 and 8.6, of 10,000
// by 2048 18.1 and 17.7.  Up to sixteen rows go this way: at sixteen tiles take 2 % less
// where the result is wide, or the contraction long, and 40 % more where neither is.
template <typename T, bool CHECK>
__device__ inline i4 piece(const T *row, int64_t k, int64_t k_end) {
    constexpr int kElems = 16 / sizeof(T);
    Piece<T, kElems> p;
    if (!CHECK || k + kElems <= k_end) {
        p.read(row + k, kElems);
    } else {
#pragma unroll
        for (int e = 0; e < kElems; ++e) p.v[e] = k + e < k_end ? row[k + e] : (T)0.f;
    }
    return __builtin_bit_cast(i4, p.v);
}

template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void rows_kernel(ProductArgs a, int by_row) {
    constexpr int kElems = 16 / sizeof(T), kSlab = 128 / sizeof(T);
    __shared__ f4 part[WAVES][64];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
    int batch = 0;
    int64_t row0 = (int64_t)blockIdx.y * 16, row_end = a.m;
    if (a.offsets) {
        const int64_t t = blockIdx.y;
        batch = expert_of(a.offsets, a.experts, by_row ? 0 : 16, t);
        const int64_t first = a.offsets[batch];
        row_end = a.offsets[batch + 1];
        row0 = by_row ? t : first + (t - (first / 16 + batch)) * 16;
        if (row0 >= row_end || (by_row && (t - first) % 16 != 0)) return;
    }
    const int64_t col0 = (int64_t)blockIdx.x * 16;
    const T *wr = static_cast<const T *>(a.b) + batch * a.batch_b +
                  (col0 + i < a.n ? col0 + i : a.n - 1) * a.ldb;
    int64_t xrow = row0 + i < row_end ? row0 + i : row_end - 1;
    if (a.list) xrow = a.per.quotient(a.list[xrow]);
    const T *xr = static_cast<const T *>(a.a) + xrow * a.lda;
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    // `count` of the wave's slabs from k on
    const auto slabs = [&](auto count, auto check, int64_t k) {
        constexpr int kCount = decltype(count)::value;
        i4 fw[kCount][2], fx[kCount][2];
#pragma unroll
        for (int s = 0; s < kCount; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = k + (int64_t)s * WAVES * kSlab + (h * 4 + g) * kElems;
                fw[s][h] = piece<T, decltype(check)::value>(wr, c, a.k);
                fx[s][h] = piece<T, decltype(check)::value>(xr, c, a.k);
            }
#pragma unroll
        for (int s = 0; s < kCount; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = multiply<T>(fw[s][h], fx[s][h], acc);
    };
    const auto fits = [&](int count, int64_t k) {
        return k + ((int64_t)(count - 1) * WAVES + 1) * kSlab <= a.k;
    };
    int64_t k = (int64_t)wave * kSlab;
    for (; fits(4, k); k += 4 * WAVES * kSlab) slabs(Int<4>(), Int<0>(), k);
    if (fits(2, k)) slabs(Int<2>(), Int<0>(), k), k += 2 * WAVES * kSlab;
    if (fits(1, k)) slabs(Int<1>(), Int<0>(), k), k += WAVES * kSlab;
    if (k < a.k) slabs(Int<1>(), Int<1>(), k);   // the last, in part
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) acc += part[w][lane];
        const int64_t row = row0 + i, col = col0 + 4 * g;
        if (row < row_end && col < a.n) {
            float u[4] = {acc[0], acc[1], acc[2], acc[3]};
            const Epilogue<T, kForward, 4> end(a, col, batch);
            typename Epilogue<T, kForward, 4>::Row extra;
            end.read(a, row, col, extra);
            end.write(row, extra, {}, u);
        }
    }
}

template <typename T, int MODE, int LIST, bool DMA, int TM, int TN, int WM, int WN>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t stream) {
    const int64_t tn = (a.n + TN - 1) / TN;
    const int64_t tm = MODE == kWeight ? (a.m + TM - 1) / TM * (a.offsets ? a.experts : 1)
                       : a.offsets     ? a.m / TM + a.experts
                                       : (a.m + TM - 1) / TM;
    if (!grid_holds(tm * tn, WM * WN * 64)) return hipErrorInvalidValue;
    constexpr int kLds = 2 * (TM + TN) * 128;
    const auto kernel = product_kernel<T, MODE, LIST, DMA, TM, TN, WM, WN>;
    if (kLds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)(tm * tn), a.splits), WM * WN * 64, kLds, stream>>>(a);
    if (MODE != kGate && a.splits > 1) {
        const int64_t quads = a.partial_rows * ((a.n + 3) / 4);
        if (!grid_holds((quads + 255) / 256, 256)) return hipErrorInvalidValue;
        join_kernel<T, MODE><<<(unsigned)((quads + 255) / 256), 256, 0, stream>>>(a, tn * TN);
    }
    return hipGetLastError();
}

// LIST: which side's rows the list names in a weight product, 1 B's, 2 A's.
template <typename T, int MODE, int LIST>
hipError_t launch_mode(const ProductArgs &a, const ProductPlan &p, hipStream_t stream) {
    if (!p.aligned)
        return p.tile == 128 ? launch_tiles<T, MODE, LIST, false, 128, 128, 2, 2>(a, stream)
                             : launch_tiles<T, MODE, LIST, false, 64, 64, 2, 2>(a, stream);
    switch (p.tile) {
        case 256: return launch_tiles<T, MODE, LIST, true, 256, 256, 2, 4>(a, stream);
        case 128: return launch_tiles<T, MODE, LIST, true, 128, 128, 2, 2>(a, stream);
        default: return launch_tiles<T, MODE, LIST, true, 64, 64, 2, 2>(a, stream);
    }
}

template <typename T, int WAVES>
hipError_t launch_rows(const ProductArgs &a, hipStream_t stream) {
    // a workgroup per 16 rows of an expert, or, with fewer rows than that could
    // make, per row, of which every sixteenth of an expert goes on
    const int64_t tiles = a.offsets ? a.m / 16 + a.experts : (a.m + 15) / 16;
    const int by_row = a.offsets && a.m < tiles;
    const int64_t high = by_row ? a.m : tiles;
    const int64_t wide = (a.n + 15) / 16;
    if (high > 65535 || !grid_holds(wide, WAVES * 64)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wide, (unsigned)high);
    rows_kernel<T, WAVES><<<grid, WAVES * 64, 0, stream>>>(a, by_row);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_product(ProductArgs a, const ProductPlan &p, hipStream_t stream) {
    a.splits = p.splits;
    switch (p.waves) {
        case 4: return launch_rows<T, 4>(a, stream);
        case 8: return launch_rows<T, 8>(a, stream);
        case 16: return launch_rows<T, 16>(a, stream);
    }
    switch (a.mode) {
        case kForward: return launch_mode<T, kForward, 0>(a, p, stream);
        case kInput: return launch_mode<T, kInput, 0>(a, p, stream);
        case kGate: return launch_mode<T, kGate, 0>(a, p, stream);
        default:
            return !a.list       ? launch_mode<T, kWeight, 0>(a, p, stream)
                   : a.list_of_a ? launch_mode<T, kWeight, 2>(a, p, stream)
                                 : launch_mode<T, kWeight, 1>(a, p, stream);
    }
}

}  // namespace
}  // namespace som
