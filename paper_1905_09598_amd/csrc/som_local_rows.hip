// Row-wise passes of the local models: operand rows copied to whole 16-byte
// pieces (with the activation's slope applied on the way where a gradient needs
// it), and the experts' answers joined per document, with their gradients.  All
// are bound by memory: each element is read and written once, 16 bytes a lane
// where the rows allow it.  dz of 16,001 x 2048 in fp16 takes 36 us (5.4 TB/s), the
// join of 8192 documents' two answers of 2048 30 us (6.8 TB/s), the sums of 16,384
// listed rows of 2048 17 us (3.9 TB/s).
#include "som_local_internal.h"

#include <algorithm>

namespace som {
namespace {

constexpr int kThreads = 256;

// N neighbouring values of a row, `left` of them there.  Rows begin at any
// element: the hardware takes 16 bytes at any address.
template <typename T, int N>
__device__ inline void read_some(const T *p, int64_t left, float (&v)[N]) {
    typedef T Vec __attribute__((ext_vector_type(N)));
    if (left >= N) {
        Vec q;
        __builtin_memcpy(&q, __builtin_assume_aligned(p, sizeof(T)), sizeof(Vec));
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)q[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = e < left ? (float)p[e] : 0.f;
    }
}
template <typename T, int N>
__device__ inline void write_some(T *p, int64_t left, const float (&v)[N]) {
    typedef T Vec __attribute__((ext_vector_type(N)));
    if (left >= N) {
        Vec q;
#pragma unroll
        for (int e = 0; e < N; ++e) q[e] = (T)v[e];
        __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T)), &q, sizeof(Vec));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < left) p[e] = (T)v[e];
    }
}

__device__ inline float slope_of(float z, int32_t kind) {
    float s;
    (void)activate(z, kind, &s);
    return s;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rows_copy_kernel(RowsArgs a) {
    constexpr int N = 16 / sizeof(T);
    const uint32_t q = blockIdx.x * kThreads + threadIdx.x, r = a.pieces.quotient(q);
    const int64_t row = r, col = (int64_t)(q - r * a.pieces.by) * N;
    if (row >= a.rows) return;
    float v[N], z[N];
    const int64_t from = a.list ? a.list[row] : row;
    read_some<T, N>(static_cast<const T *>(a.src) +
                         (a.list && from >= 0 ? (int64_t)a.per.quotient((uint32_t)from) : from) * a.lds + col,
                    from < 0 ? 0 : a.cols - col, v);
    if (a.gates) {
        const float g = from < 0 ? 0.f : a.gates[from];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = a.exponents ? ldexpf(v[e], gate_exponent(g)) : v[e] * g;
    }
    if (a.z) {
        read_some<T, N>(static_cast<const T *>(a.z) + row * a.ldz + col, a.cols - col, z);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = col + e < a.cols ? v[e] * slope_of(z[e], a.activation) : 0.f;
    }
    write_some<T, N>(static_cast<T *>(a.dst) + row * a.ldd + col, N, v);
}

// Sums of rows, in fp32 and in a fixed order: a workgroup takes 32 pieces of 16
// bytes of up to kSumRows rows of one expert (all of them if DIRECT), eight rows
// at a time, joins its eight sums a column through LDS, and writes them, or parts
// that join_sums_kernel adds up, eight at a time too.
constexpr int kSumThreads = 256, kSumPieces = 32, kSumLanes = kSumThreads / kSumPieces;
constexpr int kSumRows = 128;

template <typename T, bool DIRECT, bool LISTED>
__global__ __launch_bounds__(kSumThreads) void sums_kernel(SumsArgs a) {
    constexpr int N = 16 / sizeof(T);
    __shared__ float part[kSumLanes][kSumPieces * N + 4];
    const int piece = threadIdx.x % kSumPieces, lane = threadIdx.x / kSumPieces;
    int64_t first = (int64_t)blockIdx.x * kSumRows, end = a.rows;
    int e = 0;
    if (DIRECT) {
        e = blockIdx.x;
        first = a.offsets ? a.offsets[e] : 0;
        if (a.offsets) end = a.offsets[e + 1];
    } else {
        if (a.offsets) {
            e = expert_of(a.offsets, a.experts, kSumRows, blockIdx.x);
            first = a.offsets[e] + ((int64_t)blockIdx.x - (a.offsets[e] / kSumRows + e)) * kSumRows;
            end = a.offsets[e + 1];
        }
        end = first + kSumRows < end ? first + kSumRows : end;
        if (first >= end) return;
    }
    const int64_t col = ((int64_t)blockIdx.y * kSumPieces + piece) * N, left = a.cols - col;
    // the list's rows and weights, so that the reads of the rows wait for LDS alone
    __shared__ int row_of[LISTED && !DIRECT ? kSumRows : 1];
    __shared__ float gate_of[LISTED && !DIRECT ? kSumRows : 1];
    if (LISTED && !DIRECT) {
        const int64_t r = first + threadIdx.x;
        if (threadIdx.x < kSumRows && r < end) {
            const int slot = a.list[r];
            row_of[threadIdx.x] = a.per.quotient(slot);
            gate_of[threadIdx.x] = a.gates ? a.gates[slot] : 1.f;
        }
        __syncthreads();
    }
    float sum[N], bias[N];
#pragma unroll
    for (int c = 0; c < N; ++c) sum[c] = bias[c] = 0.f;
    if (LISTED && a.dots && left > 0)
        read_some<T, N>(static_cast<const T *>(a.bias) + e * a.cols + col, left, bias);
    constexpr int kAhead = 4;   // rows whose reads are under way together
    const int some = (int)(left < N ? left : N);
    for (int64_t r0 = first + lane; r0 < end; r0 += kAhead * kSumLanes) {
        Piece<T, N> v[kAhead];   // turned into floats when all of them are under way
        float gate[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t r = r0 + u * kSumLanes;
            int64_t row = r;
            gate[u] = 1.f;
            if (LISTED && !DIRECT && r < end) {
                row = row_of[r - first];
                gate[u] = gate_of[r - first];
            }
            if (LISTED && DIRECT && r < end) {
                const int slot = a.list[r];
                if (a.gates) gate[u] = a.gates[slot];
                row = a.per.quotient(slot);
            }
            v[u].read(static_cast<const T *>(a.src) + row * a.ld + col, r < end ? some : 0);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
#pragma unroll
            for (int c = 0; c < N; ++c)
                sum[c] = LISTED ? fmaf(gate[u], (float)v[u].v[c], sum[c]) : sum[c] + (float)v[u].v[c];
            if (LISTED && a.dots) {   // the 32 lanes of a row together
                float dot = 0.f;
#pragma unroll
                for (int c = 0; c < N; ++c) dot = fmaf((float)v[u].v[c], bias[c], dot);
#pragma unroll
                for (int o = 1; o < kSumPieces; o <<= 1) dot += __shfl_xor(dot, o);
                const int64_t r = r0 + u * kSumLanes;
                if (piece == 0 && r < end) a.dots[r * a.dot_cols + blockIdx.y] = dot;
            }
        }
    }
    if (LISTED && !a.out) return;
#pragma unroll
    for (int c = 0; c < N; ++c) part[lane][piece * N + c] = sum[c];
    __syncthreads();
    const int c = threadIdx.x;
    const int64_t at = (int64_t)blockIdx.y * kSumPieces * N + c;
    if (c < kSumPieces * N && at < a.cols) {
        float v = 0.f;
        for (int l = 0; l < kSumLanes; ++l) v += part[l][c];
        if (DIRECT) static_cast<T *>(a.out)[e * a.cols + at] = (T)v;
        else a.partial[blockIdx.x * a.cols + at] = v;
    }
}

template <typename T>
__global__ __launch_bounds__(kSumThreads) void join_sums_kernel(SumsArgs a) {
    constexpr int kCols = kSumThreads / kSumLanes;
    __shared__ float part[kSumLanes][kCols];
    const int c = threadIdx.x % kCols, lane = threadIdx.x / kCols, e = blockIdx.y;
    const int64_t col = (int64_t)blockIdx.x * kCols + c;
    int64_t first = 0, count = (a.rows + kSumRows - 1) / kSumRows;
    if (a.offsets) {
        first = a.offsets[e] / kSumRows + e;
        count = (a.offsets[e + 1] - a.offsets[e] + kSumRows - 1) / kSumRows;
    }
    float v = 0.f;
    if (col < a.cols) {
#pragma unroll 4
        for (int64_t p = lane; p < count; p += kSumLanes) v += a.partial[(first + p) * a.cols + col];
    }
    part[lane][c] = v;
    __syncthreads();
    if (lane == 0 && col < a.cols) {
        for (int l = 1; l < kSumLanes; ++l) v += part[l][c];
        static_cast<T *>(a.out)[e * a.cols + col] = (T)v;
    }
}

// 16 bytes of a document's row a thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a) {
    constexpr int N = 16 / sizeof(T);
    const uint32_t q = blockIdx.x * kThreads + threadIdx.x, r = a.pieces.quotient(q);
    const int64_t i = r, col = (int64_t)(q - r * a.pieces.by) * N, left = a.width - col;
    if (i >= a.n) return;
    float sum[N], y[N], first[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    for (int j = 0; j < a.k; ++j) {
        const int p = a.place[i * a.k + j];
        const float w = a.weight ? a.weight[i * a.k + j] : 1.f;
        if (p >= 0) {
            read_some<float, N>(a.y + p * a.width + col, left, y);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] = fmaf(w, y[e], sum[e]);
        } else if (w != w) {
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] = w;
        }
    }
    if (a.residual) {
        read_some<T, N>(static_cast<const T *>(a.residual) + i * a.ldr + col, left, first);
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += first[e];
    }
    write_some<T, N>(static_cast<T *>(a.out) + i * a.width + col, left, sum);
}

// Four lanes a slot.
template <typename T>
__global__ __launch_bounds__(kThreads) void dweight_kernel(DweightArgs a) {
    const int64_t s = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 4;
    const int lane = threadIdx.x & 3;
    const int p = s < a.slots ? a.place[s] : -1;
    float v = 0.f;
    if (p >= 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            for (int c = lane; c < a.cols[h]; c += 4) v += a.dots[h][(int64_t)p * a.cols[h] + c];
    }
    v += __shfl_xor(v, 1);
    v += __shfl_xor(v, 2);
    if (s < a.slots && lane == 0) static_cast<T *>(a.dweight)[s] = (T)v;
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

}  // namespace

// Launches `launch` on whole rows of `pieces` threads each, as many at a time as
// keep the threads' numbers below 2^31.
template <typename F>
hipError_t in_rows(int64_t rows, int64_t pieces, F launch) {
    if (pieces > INT32_MAX) return hipErrorInvalidValue;
    const int64_t most = std::max<int64_t>(1, (INT32_MAX - kThreads) / pieces);
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t some = std::min(most, rows - r);
        const hipError_t e = launch(r, some, (unsigned)((some * pieces + kThreads - 1) / kThreads));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_rows_copy(const RowsArgs &args, hipStream_t stream) {
    const int size = type_size(args.type);
    const int64_t pieces = args.ldd * size / 16;
    return in_rows(args.rows, pieces, [&](int64_t r, int64_t rows, unsigned blocks) {
        RowsArgs a = args;
        a.pieces = Divider((uint32_t)pieces);
        a.rows = rows;
        if (a.list) a.list += r;
        else a.src = static_cast<const char *>(a.src) + r * a.lds * size;
        if (a.z) a.z = static_cast<const char *>(a.z) + r * a.ldz * size;
        a.dst = static_cast<char *>(a.dst) + r * a.ldd * size;
        return by_type(a.type, [&](auto t) {
            rows_copy_kernel<decltype(t)><<<blocks, kThreads, 0, stream>>>(a);
        });
    });
}

// One pass where there are few rows.  A gradient with the sums, in one pass and in
// parts: one matrix of 2048 columns with 32, 128 and 1024 rows 13, 15, 29 and 15, 16, 19
// us; 100 experts of 512 columns with 32 and 128 rows each 23, 40 and 26, 37.  One
// pass takes as long as the most popular expert's rows, though: 4000 rows of 100 uneven
// experts 50 us longer than parts.
static bool sums_direct(const SumsArgs &a) {
    return a.rows <= (a.offsets ? (int64_t)a.experts * 16 : 128);
}
static int64_t sums_parts(const SumsArgs &a) {
    return a.offsets ? a.rows / kSumRows + a.experts : (a.rows + kSumRows - 1) / kSumRows;
}

int32_t sums_dot_cols(const SumsArgs &a) {
    const int64_t wide = 16 * kSumPieces / type_size(a.type);
    return (int32_t)((a.cols + wide - 1) / wide);
}

int64_t sums_partial(const SumsArgs &a) { return sums_direct(a) ? 0 : sums_parts(a) * a.cols; }

hipError_t launch_sums(const SumsArgs &a, hipStream_t stream) {
    const int size = type_size(a.type);
    const int experts = a.offsets ? a.experts : 1;
    const bool direct = sums_direct(a);
    const int64_t high = direct ? experts : sums_parts(a);
    const int64_t wide = (a.cols * size + 16 * kSumPieces - 1) / (16 * kSumPieces);
    if (!grid_holds(high, kSumThreads) || wide > 65535 || experts > 65535)
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)high, (unsigned)wide);
    constexpr int kCols = kSumThreads / kSumLanes;
    const dim3 join((unsigned)((a.cols + kCols - 1) / kCols), experts);
    return by_type(a.type, [&](auto t) {
        using T = decltype(t);
        if (direct) {
            if (a.list) sums_kernel<T, true, true><<<grid, kSumThreads, 0, stream>>>(a);
            else sums_kernel<T, true, false><<<grid, kSumThreads, 0, stream>>>(a);
        } else {
            if (a.list) sums_kernel<T, false, true><<<grid, kSumThreads, 0, stream>>>(a);
            else sums_kernel<T, false, false><<<grid, kSumThreads, 0, stream>>>(a);
            if (a.out) join_sums_kernel<T><<<join, kSumThreads, 0, stream>>>(a);
        }
    });
}

hipError_t launch_combine(const CombineArgs &args, hipStream_t stream) {
    const int size = type_size(args.type);
    const int64_t pieces = (args.width * size + 15) / 16;
    return in_rows(args.n, pieces, [&](int64_t r, int64_t rows, unsigned blocks) {
        CombineArgs a = args;
        a.pieces = Divider((uint32_t)pieces);
        a.n = rows;
        if (a.weight) a.weight += r * a.k;
        a.place += r * a.k;
        if (a.residual) a.residual = static_cast<const char *>(a.residual) + r * a.ldr * size;
        a.out = static_cast<char *>(a.out) + r * a.width * size;
        return by_type(a.type, [&](auto t) {
            combine_kernel<decltype(t)><<<blocks, kThreads, 0, stream>>>(a);
        });
    });
}

hipError_t launch_dweight(const DweightArgs &args, hipStream_t stream) {
    const int size = type_size(args.type);
    return in_rows(args.slots, 4, [&](int64_t s, int64_t slots, unsigned blocks) {
        DweightArgs a = args;
        a.slots = slots;
        a.place += s;
        a.dweight = static_cast<char *>(a.dweight) + s * size;
        return by_type(a.type, [&](auto t) {
            dweight_kernel<decltype(t)><<<blocks, kThreads, 0, stream>>>(a);
        });
    });
}

}  // namespace som
