// Products of matrices held in 8 bits (e4m3 with one power of two to 128 neighbours of a
// row): bringing rows to that form, the tiles of som_product.h on it, and few rows.
#include "som_product.h"

namespace som {
namespace {

constexpr int kBlock = 128;

// The power of two of a block with the largest finite magnitude `most`, as its biased
// exponent: the least e with most <= 448 2^e = 1.75 2^(8 + e), at least 2^-126.
__device__ inline int power_of(float most) {
    const uint32_t bits = __float_as_uint(most);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return e > 1 ? e : 1;
}
// 2^-(power - 127): from 2^126 down to 2^-120.
__device__ inline float one_over(int power) { return __uint_as_float((uint32_t)(254 - power) << 23); }
__device__ inline float finite_magnitude(float v) {
    const float m = fabsf(v);
    return m < INFINITY ? m : 0.f;
}
// Four values as codes, rounded to the nearest, ties to even; what is no finite number as
// the code that is none.
__device__ inline int codes_of(float a, float b, float c, float d) {
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

// Eight values of a block, of which 16 neighbouring lanes take one, as codes: from column
// `col` of a row of `width`.  Returns the block's power.
template <typename T>
__device__ inline int to_codes(const T *row, int64_t col, int64_t width, int2 *codes) {
    constexpr int N = 16 / sizeof(T);
    const int64_t left = width - col;
    float v[8], most = 0.f;
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
        const int64_t here = left - h * N;
        Piece<T, N> p;
        p.read(row + col + h * N, (int)(here < 0 ? 0 : here < N ? here : N));
#pragma unroll
        for (int e = 0; e < N; ++e) v[h * N + e] = (float)p.v[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_magnitude(v[e]));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
    const int power = power_of(most);
    const float by = one_over(power);
    codes->x = codes_of(v[0] * by, v[1] * by, v[2] * by, v[3] * by);
    codes->y = codes_of(v[4] * by, v[5] * by, v[6] * by, v[7] * by);
    return power;
}
// The powers of a wave's four blocks, 16 lanes each, as one word (in lane 0).
__device__ inline int word_of(int power) {
    return power | __shfl(power, 16) << 8 | __shfl(power, 32) << 16 | __shfl(power, 48) << 24;
}

// Bound by memory.  A wave takes four blocks of a row, 16 lanes each, eight neighbours to
// a lane, and writes their four powers as one word; the row's filling is zeros, and that
// of its powers 1.  8192 rows of 8192 in bf16 take 33 us (6.2 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void to_blocks_kernel(BlocksArgs a) {
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);   // a row's four blocks
    const uint32_t r = a.units.quotient(unit);
    if (r >= a.n) return;
    const int lane = threadIdx.x & 63;
    const int64_t row = r, block = (int64_t)(unit - r * a.units.by) * 4 + (lane >> 4);
    const int64_t col = block * kBlock + (lane & 15) * 8;
    int2 codes;
    int power = to_codes(static_cast<const T *>(a.x) + row * a.ldx, col, a.width, &codes);
    if (block * kBlock < a.width) *reinterpret_cast<int2 *>(a.codes + row * a.ld_codes + col) = codes;
    else power = 127;
    const int word = word_of(power);
    if (lane == 0)
        *reinterpret_cast<int *>(a.scale + row * a.ld_scale + block) = word;
}

// Products of up to 16 rows at a time: bound by one read of w's codes, which go straight
// from memory into the fragments.  A workgroup takes 16 columns of C, its waves four
// blocks of the contraction at a time in turn (their powers are one word), and join their
// sums through LDS in order.  CODES: x is held in 8 bits; otherwise every workgroup brings
// its rows of x to 8 bits for itself, into LDS, while its first codes of w are on their way:
// x is small, and a launch of its own would take as long as the product of one row.  One
// row of 2048 by 10,000: 7.8 us (12.1 with x brought to 8 bits by every wave in registers).
template <typename T, int WAVES, bool CODES>
__global__ __launch_bounds__(WAVES * 64) void rows8_kernel(ProductArgs a, Rows8Args b) {
    extern __shared__ __align__(16) char lds[];
    __shared__ f4 part[WAVES][64];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
    const int64_t row0 = (int64_t)blockIdx.y * 16, col0 = (int64_t)blockIdx.x * 16;
    const int rows = (int)(a.m - row0 < 16 ? a.m - row0 : 16), mine = i < rows ? i : rows - 1;
    const int64_t wrow = col0 + i < a.n ? col0 + i : a.n - 1;
    const Eight *const w = static_cast<const Eight *>(a.b) + wrow * a.ldb + g * 16;
    const unsigned char *const pw = a.scale_b + wrow * a.ld_scale;
    const int64_t blocks = a.k / kBlock;
    i4 fw[4][2];
    uint32_t word_w;
    const auto load = [&](int64_t q) {
        word_w = *reinterpret_cast<const uint32_t *>(pw + q);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (q + s < blocks) fw[s][h] = *reinterpret_cast<const i4 *>(w + (q + s) * kBlock + h * 64);
    };
    int64_t q = (int64_t)wave * 4;
    if (q < blocks) load(q);
    // x's rows, 16 bytes further apart than their codes, so that they lie on all banks
    const int64_t ldx = CODES ? a.lda : a.k + 16;
    const char *x = CODES ? static_cast<const char *>(a.a) + (row0 + mine) * ldx : lds + mine * ldx;
    const char *px = CODES ? reinterpret_cast<const char *>(a.scale_a) + (row0 + mine) * a.ld_scale
                           : lds + rows * ldx + mine * a.ld_scale;
    if constexpr (!CODES) {
        const int units = (int)(a.ld_scale / 4);   // of four blocks, of a row
        for (int u = wave; u < rows * units; u += WAVES) {
            const int r = u / units, block = (u - r * units) * 4 + (lane >> 4);
            const int64_t col = (int64_t)block * kBlock + (lane & 15) * 8;
            int2 codes;
            const int power = to_codes(static_cast<const T *>(b.x) + (row0 + r) * b.ldx, col, b.width, &codes);
            if (block < blocks) *reinterpret_cast<int2 *>(lds + r * ldx + col) = codes;
            const int word = word_of(power);
            if (lane == 0) *reinterpret_cast<int *>(lds + rows * ldx + r * a.ld_scale + block) = word;
        }
        __syncthreads();
    }
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    while (q < blocks) {
        const uint32_t word_x = *reinterpret_cast<const uint32_t *>(px + q);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (q + s >= blocks) break;   // for all alike
            const char *const from = x + (q + s) * kBlock + g * 16;
            acc = multiply_scaled(
                __builtin_shufflevector(fw[s][0], fw[s][1], 0, 1, 2, 3, 4, 5, 6, 7),
                word_w >> 8 * s & 255,
                __builtin_shufflevector(*reinterpret_cast<const i4 *>(from),
                                        *reinterpret_cast<const i4 *>(from + 64), 0, 1, 2, 3, 4, 5, 6, 7),
                word_x >> 8 * s & 255, acc);
        }
        q += WAVES * 4;
        if (q < blocks) load(q);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int v = 1; v < WAVES; ++v) acc += part[v][lane];
        const int64_t row = row0 + i, col = col0 + 4 * g;
        if (row < a.m && col < a.n) {
            float u[4] = {acc[0], acc[1], acc[2], acc[3]};
            const Epilogue<T, kForward, 4> end(a, col, 0);
            typename Epilogue<T, kForward, 4>::Row extra;
            end.read(a, row, col, extra);
            end.write(row, extra, {}, u);
        }
    }
}

template <typename T, int WAVES>
hipError_t launch_rows8(const ProductArgs &a, const Rows8Args &b, hipStream_t stream) {
    const int64_t high = (a.m + 15) / 16, wide = (a.n + 15) / 16;
    if (high > 65535 || !grid_holds(wide, WAVES * 64)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wide, (unsigned)high);
    if (b.x) rows8_kernel<T, WAVES, false><<<grid, WAVES * 64, rows8_lds(a), stream>>>(a, b);
    else rows8_kernel<T, WAVES, true><<<grid, WAVES * 64, 0, stream>>>(a, b);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(ProductArgs a, const Rows8Args &b, const ProductPlan &p, hipStream_t stream) {
    a.splits = p.splits;
    switch (p.waves) {
        case 4: return launch_rows8<T, 4>(a, b, stream);
        case 8: return launch_rows8<T, 8>(a, b, stream);
        case 16: return launch_rows8<T, 16>(a, b, stream);
    }
    switch (p.tile) {
        case 256: return launch_tiles<Eight, T, kForward, 0, true, 256, 256, 2, 4>(a, stream);
        case 128: return launch_tiles<Eight, T, kForward, 0, true, 128, 128, 2, 2>(a, stream);
        default: return launch_tiles<Eight, T, kForward, 0, true, 64, 64, 2, 2>(a, stream);
    }
}

}  // namespace

int64_t rows8_lds(const ProductArgs &a) {
    return std::min<int64_t>(a.m, 16) * (a.k + 16 + a.ld_scale);
}

hipError_t launch_product8(const ProductArgs &a, const Rows8Args &b, const ProductPlan &p,
                           hipStream_t stream) {
    return a.type == kBF16 ? launch_typed<__bf16>(a, b, p, stream)
                           : launch_typed<_Float16>(a, b, p, stream);
}

hipError_t launch_to_blocks(const BlocksArgs &args, hipStream_t stream) {
    BlocksArgs a = args;
    const int64_t units = a.ld_scale / 4, size = type_size(a.type);
    a.units = Divider((uint32_t)units);
    const int64_t most = rows_at_once(units, 4, 256);
    for (int64_t r = 0; r < args.n; r += most) {
        a.n = std::min(most, args.n - r);
        const unsigned groups = (unsigned)((a.n * units + 3) / 4);
        switch (a.type) {
            case kF32: to_blocks_kernel<float><<<groups, 256, 0, stream>>>(a); break;
            case kBF16: to_blocks_kernel<__bf16><<<groups, 256, 0, stream>>>(a); break;
            default: to_blocks_kernel<_Float16><<<groups, 256, 0, stream>>>(a); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.x = static_cast<const char *>(a.x) + a.n * a.ldx * size;
        a.codes += a.n * a.ld_codes;
        a.scale += a.n * a.ld_scale;
    }
    return hipSuccess;
}

}  // namespace som
