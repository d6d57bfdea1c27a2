// Layer norm of rows and its gradient:
//     y = (x - mean) rstd weight + bias,   rstd = 1 / sqrt(var + eps),
//     dx = rstd (g - mean(g) - xh mean(g xh)) + beside,   g = dy weight,  xh = (x - mean) rstd,
//     dweight = sum over rows of dy xh,   dbias = sum over rows of dy.
// Bound by memory: forward reads x and writes y, backward reads x and dy (and beside)
// and writes dx, once each.  A row stays in registers, 16-byte pieces of it to a lane,
// between the statistics and what they are for; rows of up to a wave's pieces are taken
// by 1 to 64 lanes, longer ones by a workgroup, and only rows beyond what a workgroup
// holds are read again.  A workgroup takes rows in turn with the weight in registers;
// backward adds up its columns' parts of dweight and dbias there, and join_parts_kernel
// adds up the workgroups' in order (no atomics: a result does not depend on timing).
// 20,000 fp16 rows of 10,000: forward 156 to 190 us (800 MB, 4.2 to 5.1 TB/s), backward
// with `beside` 289 to 310 (1.6 GB, 5.2 to 5.5 TB/s); 637 fp32 rows of 4545: 8 and 14,
// which is the reads, reductions and writes of one to three rows in turn.  5000 fp32 rows
// of 20,000, which a workgroup does not hold: 231 and 466 (with the call's second kernel).
#include "som_row.h"

#include <algorithm>

namespace som {
namespace {

template <typename T, int P, bool WIDE>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a) {
    constexpr int N = 16 / sizeof(T);
    __shared__ __align__(16) float part[kPart];
    int turn = 0;
    const Part<WIDE, P, N> me(a.lanes, (int)a.width);
    Piece<T, N> weight[P], bias[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        me.template read<T>(a.weight, 0, p, a.weight != nullptr, weight[p]);
        me.template read<T>(a.bias, 0, p, a.bias != nullptr, bias[p]);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * me.rows; r0 < a.n; r0 += (int64_t)gridDim.x * me.rows) {
        const int64_t row = r0 + me.row;
        const bool there = row < a.n;
        Piece<T, N> x[P];
#pragma unroll
        for (int p = 0; p < P; ++p) me.template read<T>(a.x, row * a.ldx, p, there, x[p]);
        float sum[1] = {0.f}, both[2] = {0.f, 0.f}, d[P][N];
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int e = 0; e < N; ++e) d[p][e] = (float)x[p].v[e];
            me.clear(p, d[p]);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[0] += d[p][e];
        }
        row_sum<WIDE>(sum, a.lanes, part, turn);
        const float m = sum[0] * a.over;
        // The mean's own rounding is found from the differences and taken out of them, so
        // that rows far from 0 keep their bits.
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int e = 0; e < N; ++e) d[p][e] = (float)x[p].v[e] - m;
            me.clear(p, d[p]);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                both[0] += d[p][e];
                both[1] = fmaf(d[p][e], d[p][e], both[1]);
            }
        }
        row_sum<WIDE>(both, a.lanes, part, turn);
        const float off = both[0] * a.over;
        const float rstd = rsqrtf(fmaxf(fmaf(-off, off, both[1] * a.over), 0.f) + a.eps);
        if (!there) continue;
        if (a.kept && me.lane == 0) {
            a.kept[2 * row] = m + off;
            a.kept[2 * row + 1] = rstd;
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            Piece<T, N> y;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float v = ((float)x[p].v[e] - m - off) * rstd;
                if (a.weight) v *= (float)weight[p].v[e];
                if (a.bias) v += (float)bias[p].v[e];
                y.v[e] = (T)v;
            }
            if (me.mine(p)) y.write(static_cast<T *>(a.y) + row * a.width + me.at[p], N);
        }
    }
}

// Rows that a workgroup does not hold, and rows shorter than a piece: read three times,
// the later ones mostly from the caches.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
    constexpr int N = 16 / sizeof(T);
    __shared__ __align__(16) float part[kPart];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *const x = static_cast<const T *>(a.x) + row * a.ldx;
        float sum[1] = {0.f}, both[2] = {0.f, 0.f};
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.width; c += (int64_t)blockDim.x * N) {
            Piece<T, N> v;
            v.read(x + c, (int)std::min<int64_t>(N, a.width - c));
#pragma unroll
            for (int e = 0; e < N; ++e) sum[0] += (float)v.v[e];
        }
        row_sum<true>(sum, 0, part, turn);
        const float m = sum[0] * a.over;
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.width; c += (int64_t)blockDim.x * N) {
            const int left = (int)std::min<int64_t>(N, a.width - c);
            Piece<T, N> v;
            v.read(x + c, left);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float d = e < left ? (float)v.v[e] - m : 0.f;
                both[0] += d;
                both[1] = fmaf(d, d, both[1]);
            }
        }
        row_sum<true>(both, 0, part, turn);
        const float off = both[0] * a.over;
        const float rstd = rsqrtf(fmaxf(fmaf(-off, off, both[1] * a.over), 0.f) + a.eps);
        if (a.kept && threadIdx.x == 0) {
            a.kept[2 * row] = m + off;
            a.kept[2 * row + 1] = rstd;
        }
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.width; c += (int64_t)blockDim.x * N) {
            const int left = (int)std::min<int64_t>(N, a.width - c);
            Piece<T, N> v, weight, bias;
            v.read(x + c, left);
            if (a.weight) weight.read(static_cast<const T *>(a.weight) + c, left);
            if (a.bias) bias.read(static_cast<const T *>(a.bias) + c, left);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float u = ((float)v.v[e] - m - off) * rstd;
                if (a.weight) u *= (float)weight.v[e];
                if (a.bias) u += (float)bias.v[e];
                v.v[e] = (T)u;
            }
            v.write(static_cast<T *>(a.y) + row * a.width + c, left);
        }
    }
}

// What backward's sums of a row give: of g, of g (x - mean), of x - mean.  kept holds the
// mean as fp32 rounds it, so what the differences from it add up to is taken out again, as
// forward does: the gradients of rows far from 0 keep their bits.  With xh of the rounded mean,
//     dx = rstd (g - level - xh slope) + beside,    dweight = sum of dy (xh - off).
struct Shares {
    float off, slope, level;
    __device__ Shares(const float (&sums)[3], float rstd, float over) {
        const float g = sums[0] * over;
        off = sums[2] * over * rstd;
        slope = sums[1] * over * rstd - off * g;
        level = g - off * slope;
    }
};

// COLUMNS: also the workgroup's parts of dweight and dbias.  AHEAD: a row's reads are on
// their way while the one before it is worked on; that takes the registers of a larger
// workgroup than kAheadThreads.
constexpr int kAheadThreads = 768;
template <typename T, int P, bool WIDE, bool COLUMNS, bool AHEAD>
__global__ __launch_bounds__(AHEAD ? kAheadThreads : 1024) void norm_backward_kernel(NormArgs a) {
    constexpr int N = 16 / sizeof(T);
    extern __shared__ __align__(16) float lds[];
    float *const part = lds;          // kPart
    int turn = 0;
    const Part<WIDE, P, N> me(a.lanes, (int)a.width);
    Piece<T, N> weight[P];
    float dweight[P][N], dbias[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        me.template read<T>(a.weight, 0, p, a.weight != nullptr, weight[p]);
#pragma unroll
        for (int e = 0; e < N; ++e) dweight[p][e] = dbias[p][e] = 0.f;
    }
    const int64_t step = (int64_t)gridDim.x * me.rows;
    struct Row {
        Piece<T, N> x[P], dy[P], beside[P];
        float mean, rstd;
    } next;
    const auto read = [&](int64_t row, Row &to) {
        const bool there = row < a.n;
        to.mean = there ? a.kept[2 * row] : 0.f;
        to.rstd = there ? a.kept[2 * row + 1] : 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            me.template read<T>(a.x, row * a.ldx, p, there, to.x[p]);
            me.template read<T>(a.dy, row * a.lddy, p, there, to.dy[p]);
            if (a.beside) me.template read<T>(a.beside, row * a.ldb, p, there, to.beside[p]);
        }
    };
    if (AHEAD) read((int64_t)blockIdx.x * me.rows + me.row, next);
    for (int64_t r0 = (int64_t)blockIdx.x * me.rows; r0 < a.n; r0 += step) {
        const int64_t row = r0 + me.row;
        const bool there = row < a.n;
        Row here;
        if (AHEAD) {
            here = next;
            read(row + step, next);
        } else {
            read(row, here);
        }
        auto &x = here.x, &dy = here.dy;
        const auto &beside = here.beside;
        const float mean = here.mean, rstd = here.rstd;
        float sums[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float u[N], d[N];
#pragma unroll
            for (int e = 0; e < N; ++e) u[e] = (float)dy[p].v[e], d[e] = (float)x[p].v[e] - mean;
            me.clear(p, u);
            me.clear(p, d);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float g = a.weight ? u[e] * (float)weight[p].v[e] : u[e];
                sums[0] += g;
                sums[1] = fmaf(g, d[e], sums[1]);
                sums[2] += d[e];
            }
            // fp32's pieces one after the other: three of them together take more registers
            // than there are (20,000 rows of 4545: 270 us, so 224)
            if (sizeof(T) == 4) asm volatile("" : "+v"(sums[0]), "+v"(sums[1]), "+v"(sums[2]));
        }
        row_sum<WIDE>(sums, a.lanes, part, turn);
        keep_raw<T, P>(x);
        keep_raw<T, P>(dy);
        if (!there) continue;
        const Shares s(sums, rstd, a.over);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            Piece<T, N> dx;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float u = (float)dy[p].v[e];
                const float xh = ((float)x[p].v[e] - mean) * rstd;
                if (COLUMNS) {
                    dweight[p][e] = fmaf(u, xh - s.off, dweight[p][e]);
                    dbias[p][e] += u;
                }
                const float g = a.weight ? u * (float)weight[p].v[e] : u;
                float v = rstd * (g - s.level - xh * s.slope);
                if (a.beside) v += (float)beside[p].v[e];
                dx.v[e] = (T)v;
            }
            if (a.dx && me.mine(p)) dx.write(static_cast<T *>(a.dx) + row * a.width + me.at[p], N);
        }
    }
    if (!COLUMNS) return;
    float *const to = a.partial + (int64_t)blockIdx.x * 2 * a.width;
    if (WIDE) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (e >= me.skip[p]) {
                    to[me.at[p] + e] = dweight[p][e];
                    to[a.width + me.at[p] + e] = dbias[p][e];
                }
            }
        return;
    }
    // the rows of a wave by exchange, the four waves through LDS: each column's two sums
    float *const shared = lds + kPart;   // 4 x width x 2
    const int wave = threadIdx.x >> 6, span = (int)a.width * 2;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            for (int o = a.lanes; o < 64; o <<= 1) {
                dweight[p][e] += __shfl_xor(dweight[p][e], o);
                dbias[p][e] += __shfl_xor(dbias[p][e], o);
            }
            if ((threadIdx.x & 63) < a.lanes && e >= me.skip[p]) {
                float *const at = shared + wave * span + (me.at[p] + e) * 2;
                at[0] = dweight[p][e];
                at[1] = dbias[p][e];
            }
        }
    __syncthreads();
    for (int c = threadIdx.x; c < span; c += blockDim.x) {
        float v = 0.f;
        for (int w = 0; w < 4; ++w) v += shared[w * span + c];
        to[(c & 1) * a.width + (c >> 1)] = v;
    }
}

// dx of such rows, and what their means are off for their columns' sums.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_backward_kernel(NormArgs a) {
    constexpr int N = 16 / sizeof(T);
    __shared__ __align__(16) float part[kPart];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *const x = static_cast<const T *>(a.x) + row * a.ldx;
        const T *const dy = static_cast<const T *>(a.dy) + row * a.lddy;
        const float mean = a.kept[2 * row], rstd = a.kept[2 * row + 1];
        const auto values = [&](int64_t c, int left, float (&g)[N], float (&d)[N]) {
            Piece<T, N> u, v, weight;
            u.read(dy + c, left);
            v.read(x + c, left);
            if (a.weight) weight.read(static_cast<const T *>(a.weight) + c, left);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                g[e] = a.weight ? (float)u.v[e] * (float)weight.v[e] : (float)u.v[e];
                d[e] = e < left ? (float)v.v[e] - mean : 0.f;
            }
        };
        float sums[3] = {0.f, 0.f, 0.f}, g[N], d[N];
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.width; c += (int64_t)blockDim.x * N) {
            values(c, (int)std::min<int64_t>(N, a.width - c), g, d);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sums[0] += g[e];
                sums[1] = fmaf(g[e], d[e], sums[1]);
                sums[2] += d[e];
            }
        }
        row_sum<true>(sums, 0, part, turn);
        const Shares s(sums, rstd, a.over);
        if (a.off && threadIdx.x == 0) a.off[row] = s.off;
        if (!a.dx) continue;
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.width; c += (int64_t)blockDim.x * N) {
            const int left = (int)std::min<int64_t>(N, a.width - c);
            values(c, left, g, d);
            Piece<T, N> beside, dx;
            if (a.beside) beside.read(static_cast<const T *>(a.beside) + row * a.ldb + c, left);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float v = rstd * (g[e] - s.level - d[e] * rstd * s.slope);
                if (a.beside) v += (float)beside.v[e];
                dx.v[e] = (T)v;
            }
            dx.write(static_cast<T *>(a.dx) + row * a.width + c, left);
        }
    }
}

// Their parts of dweight and dbias, 256 pieces of a row to a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a) {
    constexpr int N = 16 / sizeof(T);
    const int64_t col = ((int64_t)blockIdx.y * 256 + threadIdx.x) * N;
    if (col >= a.width) return;
    const int left = (int)std::min<int64_t>(N, a.width - col);
    float dweight[N], dbias[N];
#pragma unroll
    for (int e = 0; e < N; ++e) dweight[e] = dbias[e] = 0.f;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const float mean = a.kept[2 * row], rstd = a.kept[2 * row + 1], off = a.off[row];
        Piece<T, N> u, v;
        u.read(static_cast<const T *>(a.dy) + row * a.lddy + col, left);
        v.read(static_cast<const T *>(a.x) + row * a.ldx + col, left);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            dweight[e] = fmaf((float)u.v[e], ((float)v.v[e] - mean) * rstd - off, dweight[e]);
            dbias[e] += (float)u.v[e];
        }
    }
    float *const to = a.partial + (int64_t)blockIdx.x * 2 * a.width + col;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < left) {
            to[e] = dweight[e];
            to[a.width + e] = dbias[e];
        }
}

// Two rows of `width` from their parts, in order: four neighbouring columns a thread, 32 of
// them to a workgroup, the parts in turn over 32 lanes (512 parts of 8192: 6 us).
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const float *partial, int32_t parts,
                                                         int64_t width, T *first, T *second) {
    constexpr int kLanes = 32, kQuads = 256 / kLanes;
    __shared__ float part[kLanes][4 * kQuads + 1];
    const int q = threadIdx.x % kQuads, lane = threadIdx.x / kQuads;
    const int64_t from = ((int64_t)blockIdx.x * kQuads + q) * 4, left = 2 * width - from;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = lane; p < parts; p += kLanes) {
        Piece<float, 4> u;
        u.read(partial + p * 2 * width + from, (int)(left < 0 ? 0 : left < 4 ? left : 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u.v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) part[lane][4 * q + e] = v[e];
    __syncthreads();
    const int c = threadIdx.x;
    const int64_t col = (int64_t)blockIdx.x * kQuads * 4 + c;
    if (c < 4 * kQuads && col < 2 * width) {
        float sum = 0.f;
        for (int l = 0; l < kLanes; ++l) sum += part[l][c];
        T *const to = col < width ? first : second;
        if (to) to[col < width ? col : col - width] = (T)sum;
    }
}

// Pieces that a lane has registers for (a workgroup of 1024 threads has 128 for each).
constexpr int kWavePieces = 2;
template <typename T>
constexpr int kForwardPieces = sizeof(T) == 4 ? 4 : 2;
template <typename T>
constexpr int kBackwardPieces = sizeof(T) == 4 ? 3 : 2;
Shape forward_shape(const NormArgs &a) {
    return shape_of(a.type, a.width, kWavePieces,
                    a.type == kF32 ? kForwardPieces<float> : kForwardPieces<__bf16>, 256);
}
Shape backward_shape(const NormArgs &a) {
    return shape_of(a.type, a.width, kWavePieces,
                    a.type == kF32 ? kBackwardPieces<float> : kBackwardPieces<__bf16>, 256);
}

constexpr int64_t kPartRows = 3;

// Workgroups of a launch of row after row: as many as run at a time, of `waves` waves to a
// compute unit.  More of them, which have to wait, read worse (20,000 fp16 rows of 10,000,
// two workgroups to a compute unit 165 us, three 189, a row each 216).
int64_t groups_of(const NormArgs &a, const Shape &s, int waves, int num_cus) {
    const int64_t rows = s.held && !s.wide ? s.threads / s.lanes : 1;
    const int64_t fit = std::max(1, waves * 64 / s.threads);
    return std::min((a.n + rows - 1) / rows, num_cus * fit);
}
// Waves that a compute unit holds, by the registers that a row's values take.
int forward_waves(const NormArgs &a, const Shape &s) {
    const int values = s.pieces * (16 / type_size(a.type));
    return values <= 8 ? 32 : a.type == kF32 && values > 12 ? 20 : 24;
}
int backward_waves(const Shape &s) { return s.pieces <= 1 ? 20 : 12; }

}  // namespace

// Groups of rows whose parts of dweight and dbias are added up apart: the workgroups, each
// of kPartRows rows or more.
int32_t norm_parts(const NormArgs &a, int num_cus) {
    const Shape s = backward_shape(a);
    const int64_t rows = s.held && !s.wide ? s.threads / s.lanes : 1;
    const int64_t groups = s.held ? std::min(groups_of(a, s, backward_waves(s), num_cus),
                                             (a.n + kPartRows * rows - 1) / (kPartRows * rows))
                                  : std::min<int64_t>((a.n + 15) / 16, num_cus);
    return (int32_t)std::max<int64_t>(1, groups);
}

bool norm_long_columns(const NormArgs &a) { return !backward_shape(a).held && (a.dweight || a.dbias); }

hipError_t launch_join_parts(int32_t type, const float *partial, int32_t parts, int64_t width,
                             void *first, void *second, hipStream_t stream) {
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        join_parts_kernel<T><<<(unsigned)((2 * width + 31) / 32), 256, 0, stream>>>(
            partial, parts, width, static_cast<T *>(first), static_cast<T *>(second));
    });
}

hipError_t launch_norm(const NormArgs &args, int num_cus, hipStream_t stream) {
    NormArgs a = args;
    const Shape s = forward_shape(a);
    const unsigned groups = (unsigned)groups_of(a, s, s.held ? forward_waves(a, s) : 32, num_cus);
    a.lanes = s.lanes;
    a.over = 1.f / (float)a.width;
    return by_type(a.type, [&](auto t) {
        using T = decltype(t);
        if (!s.held) {
            norm_long_kernel<T><<<groups, s.threads, 0, stream>>>(a);
            return;
        }
        by_pieces<kForwardPieces<T>>(s.pieces, [&](auto p) {
            constexpr int P = decltype(p)::value;
            if (s.wide) norm_kernel<T, P, true><<<groups, s.threads, 0, stream>>>(a);
            else norm_kernel<T, P, false><<<groups, s.threads, 0, stream>>>(a);
        });
    });
}

hipError_t launch_norm_backward(const NormArgs &args, int num_cus, hipStream_t stream) {
    NormArgs a = args;
    const Shape s = backward_shape(a);
    const bool columns = a.dweight || a.dbias;
    a.lanes = s.lanes;
    a.over = 1.f / (float)a.width;
    const unsigned groups = columns ? (unsigned)a.parts : (unsigned)groups_of(a, s, backward_waves(s), num_cus);
    const int64_t wide = (a.width * type_size(a.type) + 16 * 256 - 1) / (16 * 256);
    const hipError_t e = by_type(a.type, [&](auto t) {
        using T = decltype(t);
        if (s.held) {
            by_pieces<kBackwardPieces<T>>(s.pieces, [&](auto p) {
                constexpr int P = decltype(p)::value;
                const unsigned lds =
                    (unsigned)((kPart + (columns && !s.wide ? 4 * a.width * 2 : 0)) * sizeof(float));
                const auto launch = [&](auto wide, auto cols, auto ahead) {
                    norm_backward_kernel<T, P, decltype(wide)::value, decltype(cols)::value,
                                         decltype(ahead)::value><<<groups, s.threads, lds, stream>>>(a);
                };
                const auto by_columns = [&](auto wide, auto ahead) {
                    if (columns) launch(wide, Int<1>(), ahead);
                    else launch(wide, Int<0>(), ahead);
                };
                if (!s.wide) by_columns(Int<0>(), Int<1>());
                else if (s.threads <= kAheadThreads) by_columns(Int<1>(), Int<1>());
                else by_columns(Int<1>(), Int<0>());
            });
        } else {
            const unsigned rows = (unsigned)groups_of(a, s, 32, num_cus);
            if (a.n) norm_long_backward_kernel<T><<<rows, s.threads, 0, stream>>>(a);
            if (columns)
                norm_columns_kernel<T><<<dim3(groups, (unsigned)wide), 256, 0, stream>>>(a);
        }
    });
    if (e != hipSuccess || !columns) return e;
    return launch_join_parts(a.type, a.partial, a.parts, a.width, a.dweight, a.dbias, stream);
}

}  // namespace som
