// The pass between the gradient of a gated layer y = act(u) v and the products for its
// input's and its matrices' gradients:
//     dz = [ dy v act'(u)    dy act(u) ]
// and the sums of dz's columns, from fp32 u and v as forward kept them (in 16 bits their
// roundings would reach all of the gradient: errors of 1.8 times one rounding, 1.4 as it
// is).  Bound by memory: 2 reads of 4 bytes, one of dy, two writes to each.  A thread
// keeps to its columns, 16 bytes of dy, and goes down a group of rows with the sums of
// its columns in registers; the groups' sums are joined in order (som_norm.hip).  dz is
// rounded to the element type for the matrix instructions, the sums are of dz before that.
// 8192 x 4096 in bf16: 113 us (4.2 TB/s).
// fp16 does not hold all of dz's range, where the gradients of x and w may be ordinary
// numbers: dy v can pass 65,520 where neither does, and dy of a mean's loss begins next to
// its subnormals.  There the pass keeps its largest magnitude too, and a second launch, which
// otherwise only looks, writes dz once more over a power of two where that is outside
// [1/4, 65,520); the products take the power to their sums.  2 to 4 us where it only looks,
// 85 of 8192 x 4096 where it writes.
#include "som_local_internal.h"

#include <algorithm>
#include <type_traits>

namespace som {
namespace {

constexpr int kThreads = 256;

// Threads of a workgroup that share a group of rows, a power of two: rows of few columns
// leave room for several groups.
__host__ __device__ inline int lanes_of(const GatedArgs &a) {
    const int n = a.type == kF32 ? 4 : 8;
    int lanes = 1;
    while (lanes < kThreads && (int64_t)lanes * n < a.hidden) lanes *= 2;
    return lanes;
}

// The power of two by which dz of this largest magnitude is held in fp16: with it the
// largest lies in [2^14, 2^15), without it elements keep all bits down to 2^-12 of it.
__device__ inline int held_power(float largest) {
    return largest == 0.f || (largest >= 0.25f && largest < 65520.f)
               ? 0
               : __builtin_amdgcn_frexp_expf(largest) - 15;
}

// The largest of the workgroup's values, in all of its threads.
__device__ inline float group_max(float v) {
    __shared__ float part[kThreads / 64];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) v = fmaxf(v, part[w]);
    return v;
}

// AGAIN: dz alone, over the power of two that its largest magnitude asks for.
template <typename T, bool AGAIN>
__global__ __launch_bounds__(kThreads) void gated_slopes_kernel(GatedArgs a) {
    constexpr int N = 16 / sizeof(T), kAhead = 2;   // rows whose reads are under way together
    constexpr bool kHalf = std::is_same<T, _Float16>::value;
    const int64_t group = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    float largest = 0.f;
    int power = 0;
    if (AGAIN) {
        for (int64_t i = threadIdx.x; i < (int64_t)gridDim.x * gridDim.y; i += kThreads)
            largest = fmaxf(largest, a.largest[i]);
        power = held_power(group_max(largest));
        if (group == 0 && threadIdx.x == 0) *a.power = power;
        if (power == 0) return;
    }
    const int lanes = lanes_of(a), rows = kThreads / lanes;
    const int64_t part = (int64_t)blockIdx.x * rows + threadIdx.x / lanes;   // group of rows
    int64_t col = ((int64_t)blockIdx.y * lanes + threadIdx.x % lanes) * N;
    const bool there = col < a.hidden && part < a.parts;
    if (!there && (AGAIN || !kHalf)) return;
    const bool last = col + N >= a.hidden;
    const int left = a.hidden < N ? (int)a.hidden : N;
    // A piece that crosses the row's end begins earlier, so that its reads are whole; the
    // first `skip` columns are the piece's before it too, which writes the same there.
    const int skip = last && a.hidden >= N ? (int)(col + N - a.hidden) : 0;
    col -= skip;
    float sum[2][N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[0][e] = sum[1][e] = 0.f;
    for (int64_t r0 = there ? part : a.n; r0 < a.n; r0 += (int64_t)a.parts * kAhead) {
        Piece<T, N> dy[kAhead];
        Piece<float, N> z[kAhead][2];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int64_t r = r0 + (int64_t)q * a.parts;
            const int some = r < a.n ? left : 0;
            dy[q].read(static_cast<const T *>(a.dy) + r * a.lddy + col, some);
            z[q][0].read(a.z + r * 2 * a.hidden + col, some);
            z[q][1].read(a.z + (r * 2 + 1) * a.hidden + col, some);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int64_t r = r0 + (int64_t)q * a.parts;
            if (r >= a.n) break;
            Piece<T, N> out[2];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float slope;
                const float act = activate(z[q][0].v[e], a.activation, &slope);
                const float d = (float)dy[q].v[e], du = d * z[q][1].v[e] * slope, dv = d * act;
                sum[0][e] += du;
                sum[1][e] += dv;
                out[0].v[e] = (T)(AGAIN ? __builtin_amdgcn_ldexpf(du, -power) : du);
                out[1].v[e] = (T)(AGAIN ? __builtin_amdgcn_ldexpf(dv, -power) : dv);
                if (kHalf && !AGAIN) {
                    const float u = fabsf(du), v = fabsf(dv);
                    largest = fmaxf(largest, u < INFINITY ? u : 0.f);
                    largest = fmaxf(largest, v < INFINITY ? v : 0.f);
                }
            }
            T *const to = static_cast<T *>(a.dz) + r * a.ldd + col;
            out[0].write(to, left);
            out[1].write(to + a.hidden, left);
            if (last)                       // the row's filling
                for (int64_t c = 2 * a.hidden; c < a.ldd; ++c)
                    static_cast<T *>(a.dz)[r * a.ldd + c] = (T)0.f;
        }
    }
    if (AGAIN) return;
    if (kHalf) {
        largest = group_max(largest);
        if (threadIdx.x == 0) a.largest[group] = largest;
    }
    if (!a.partial || !there) return;
    float *const to = a.partial + part * 2 * a.hidden + col;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e >= skip && e < left) {
            to[e] = sum[0][e];
            to[a.hidden + e] = sum[1][e];
        }
}

int64_t wide_of(const GatedArgs &a) {
    return (a.hidden * type_size(a.type) + 16 * kThreads - 1) / (16 * kThreads);
}

}  // namespace

// Groups of rows: of as many threads as two workgroups to a compute unit have, and two
// rows or more to a group (8192 x 4096 in bf16 with the join of the sums: two 117 us, four
// 122, eight 128, sixteen 146).
int32_t gated_parts(const GatedArgs &a, int num_cus) {
    const int64_t rows = kThreads / lanes_of(a);
    const int64_t most = std::max<int64_t>(1, (int64_t)num_cus * 2 / wide_of(a)) * rows;
    return (int32_t)std::max<int64_t>(1, std::min(most, (a.n + 1) / 2));
}

int64_t gated_largest(const GatedArgs &a) {
    if (a.type != kF16) return 0;
    const int64_t rows = kThreads / lanes_of(a);
    return (a.parts + rows - 1) / rows * wide_of(a);
}

hipError_t launch_gated_slopes(const GatedArgs &a, hipStream_t stream) {
    const int rows = kThreads / lanes_of(a);
    const dim3 grid((unsigned)((a.parts + rows - 1) / rows), (unsigned)wide_of(a));
    switch (a.type) {
        case kF32: gated_slopes_kernel<float, false><<<grid, kThreads, 0, stream>>>(a); break;
        case kBF16: gated_slopes_kernel<__bf16, false><<<grid, kThreads, 0, stream>>>(a); break;
        default: {
            gated_slopes_kernel<_Float16, false><<<grid, kThreads, 0, stream>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            gated_slopes_kernel<_Float16, true><<<grid, kThreads, 0, stream>>>(a);
        }
    }
    return hipGetLastError();
}

}  // namespace som
