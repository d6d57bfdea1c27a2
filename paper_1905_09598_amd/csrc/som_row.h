// Rows in registers: what layer norm and distillation share.  A row lies in 16-byte
// pieces, P to a lane, over 1 to 64 neighbouring lanes or (WIDE) a whole workgroup.
#pragma once

#include "som_local_internal.h"

#include <type_traits>

namespace som {
namespace {

// Room in LDS for what a workgroup's waves exchange: two halves, of which exchanges in
// turn take one and the other, so that one barrier each will do.
constexpr int kPartValues = 4, kPart = 2 * 16 * kPartValues;

// Joins VALUES values over the lanes of a row: `lanes` neighbours (a power of two), or
// with WIDE the whole workgroup, in the same order for every lane.  The values' exchanges
// are under way together; a wave's lie side by side and are read as one (of four waves
// ahead: of eight they take 16 registers more).
template <bool WIDE, int VALUES, typename F>
__device__ inline void row_join(float (&v)[VALUES], int lanes, float *part, int &turn, F join) {
    static_assert(VALUES <= kPartValues, "room for them");
    constexpr int kRoom = VALUES == 3 ? 4 : VALUES;
    typedef float Values __attribute__((ext_vector_type(kRoom)));
    for (int o = 1; o < (WIDE ? 64 : lanes); o <<= 1) {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) v[i] = join(v[i], __shfl_xor(v[i], o));
    }
    if (!WIDE) return;
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
    Values *const mine = reinterpret_cast<Values *>(part) + (turn ^= 1) * (kPart / 2 / kRoom);
    if ((threadIdx.x & 63) == 0) {
        Values all = {};
#pragma unroll
        for (int i = 0; i < VALUES; ++i) all[i] = v[i];
        mine[wave] = all;
    }
    __syncthreads();
    Values all = mine[0];
#pragma unroll
    for (int i = 0; i < VALUES; ++i) v[i] = all[i];
#pragma unroll 4
    for (int w = 1; w < waves; ++w) {
        all = mine[w];
#pragma unroll
        for (int i = 0; i < VALUES; ++i) v[i] = join(v[i], all[i]);
    }
}
template <bool WIDE, int VALUES>
__device__ inline void row_sum(float (&v)[VALUES], int lanes, float *part, int &turn) {
    row_join<WIDE>(v, lanes, part, turn, [](float a, float b) { return a + b; });
}
template <bool WIDE, int VALUES>
__device__ inline void row_max(float (&v)[VALUES], int lanes, float *part, int &turn) {
    row_join<WIDE>(v, lanes, part, turn, [](float a, float b) { return fmaxf(a, b); });
}

// A thread's part of a row of at least N elements: P pieces of N neighbours.  A piece
// that crosses the row's end begins earlier instead, so that every read is whole: its
// first `skip` elements belong to the piece before it, are left out of sums, and are
// written by both alike.  A piece that begins beyond the end has skip = N.
template <bool WIDE, int P, int N>
struct Part {
    int lane, row, rows;   // its place among the row's lanes; its row of the workgroup's `rows`
    int at[P], skip[P];
    __device__ Part(int lanes, int width) {
        lane = WIDE ? threadIdx.x : threadIdx.x & (lanes - 1);
        row = WIDE ? 0 : threadIdx.x / lanes;
        rows = WIDE ? 1 : blockDim.x / lanes;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (lane + p * lanes) * N;
            at[p] = col + N <= width ? col : width - N;
            skip[p] = col - at[p] < N ? col - at[p] : N;
        }
    }
    __device__ bool mine(int p) const { return skip[p] < N; }
    // 0 in place of what belongs to another piece.
    __device__ void clear(int p, float (&v)[N]) const {
        if (skip[p] > 0) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = e < skip[p] ? 0.f : v[e];
        }
    }
    template <typename T>
    __device__ void read(const void *rows_at, int64_t first, int p, bool there, Piece<T, N> &v) const {
        if (there && mine(p)) v.read(static_cast<const T *>(rows_at) + first + at[p], N);
        else v.read(nullptr, 0);
    }
};

// Keeps a row's pieces as they were read between its passes, not the floats that the last
// pass made of them, which would take more registers than there are.
template <typename T, int P>
__device__ inline void keep_raw(Piece<T, 16 / sizeof(T)> (&x)[P]) {
    typedef int Raw __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int p = 0; p < P; ++p) {
        Raw raw = __builtin_bit_cast(Raw, x[p].v);
        asm volatile("" : "+v"(raw));
        x[p].v = __builtin_bit_cast(decltype(x[p].v), raw);
    }
}

// How rows are taken: pieces to a lane, lanes to a row, threads of a workgroup.
struct Shape {
    int pieces, lanes, threads;
    bool wide, held;
};

// most_wave, most_wide: pieces that a lane has registers for, of a row that a few lanes
// take and of one that a workgroup takes; threads: of a workgroup that takes several rows.
inline Shape shape_of(int32_t type, int64_t width, int most_wave, int most_wide, int threads) {
    const int n = 16 / type_size(type);
    const int64_t pieces = (width + n - 1) / n;
    Shape s{};
    s.wide = pieces > 64 * most_wave;
    s.held = pieces <= (int64_t)1024 * most_wide && width >= n;
    if (!s.held) {
        s.threads = width < n ? 64 : 1024;
    } else if (!s.wide) {
        s.pieces = (int)(pieces + 63) / 64;
        s.lanes = 1;
        while (s.lanes * s.pieces < pieces) s.lanes *= 2;
        s.threads = threads;
    } else {
        s.pieces = most_wide;
        s.lanes = (int)((pieces + 64 * s.pieces - 1) / (64 * s.pieces)) * 64;
        // as few pieces to a lane as these lanes allow
        while (s.pieces > 1 && (int64_t)s.lanes * (s.pieces - 1) >= pieces) --s.pieces;
        s.threads = s.lanes;
    }
    return s;
}

template <typename F>
hipError_t by_type(int32_t type, F f) {
    switch (type) {
        case kF32: f(float()); break;
        case kBF16: f(__bf16()); break;
        default: f(_Float16()); break;
    }
    return hipGetLastError();
}

template <int V>
using Int = std::integral_constant<int, V>;

// f(Int<pieces>()), of up to MOST.
template <int MOST, typename F>
void by_pieces(int pieces, F f) {
    if constexpr (MOST > 1) {
        if (pieces < MOST) return by_pieces<MOST - 1>(pieces, f);
    }
    f(Int<MOST>());
}

}  // namespace
}  // namespace som
