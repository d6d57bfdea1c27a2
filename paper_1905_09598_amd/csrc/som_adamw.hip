// AdamW over many tensors in one launch (som_local.h has the formulas).  A
// workgroup takes up to 2048 neighbouring elements of one tensor, its four waves
// blocks of 256 in turn: four elements a lane, so a block's largest magnitude is a
// reduction over one wave.  A table made once names each workgroup's tensor; the
// gradients' addresses come with the launch.  Bound by memory: 67M elements in
// bf16 with masters and 8-bit states, 1.08 GB, take 200 us (5.4 TB/s).
//
// The arithmetic is fp32, each operation rounded by itself (the translation unit
// is compiled without contraction), so that the codes of 8-bit states do not
// depend on which operations a compiler fuses.
#include "som_local_internal.h"

#include <math.h>

namespace som {
namespace {

constexpr int kThreads = 256;

// Four neighbours of a packed array, `left` of them there.  Arrays begin at any
// element: the hardware takes 16 bytes at any address.
template <typename T>
__device__ inline void read_typed(const void *p, int64_t at, int left, float (&v)[4]) {
    typedef T Vec __attribute__((ext_vector_type(4)));
    const T *from = static_cast<const T *>(p) + at;
    if (left >= 4) {
        Vec q;
        __builtin_memcpy(&q, __builtin_assume_aligned(from, sizeof(T)), sizeof(Vec));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)q[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < left ? (float)from[e] : 0.f;
    }
}
template <typename T>
__device__ inline void write_typed(void *p, int64_t at, int left, const float (&v)[4]) {
    typedef T Vec __attribute__((ext_vector_type(4)));
    T *to = static_cast<T *>(p) + at;
    if (left >= 4) {
        Vec q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = (T)v[e];
        __builtin_memcpy(__builtin_assume_aligned(to, sizeof(T)), &q, sizeof(Vec));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) to[e] = (T)v[e];
    }
}
__device__ inline void read_any(int type, const void *p, int64_t at, int left, float (&v)[4]) {
    if (type == kF32) read_typed<float>(p, at, left, v);
    else if (type == kBF16) read_typed<__bf16>(p, at, left, v);
    else read_typed<_Float16>(p, at, left, v);
}
__device__ inline void write_any(int type, void *p, int64_t at, int left, const float (&v)[4]) {
    if (type == kF32) write_typed<float>(p, at, left, v);
    else if (type == kBF16) write_typed<__bf16>(p, at, left, v);
    else write_typed<_Float16>(p, at, left, v);
}

// Largest magnitude over the wave; a NaN is larger than all (its bits are).
__device__ inline float wave_top(const float (&v)[4]) {
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    return __uint_as_float(top);
}

__device__ inline unsigned to_codes(const float (&v)[4]) {
    int q = 0;
    q = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], q, false);
    q = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], q, true);
    return (unsigned)q;
}
__device__ inline void from_codes(unsigned q, float scale, float (&v)[4]) {
    v[0] = __builtin_amdgcn_cvt_f32_fp8(q, 0) * scale;
    v[1] = __builtin_amdgcn_cvt_f32_fp8(q, 1) * scale;
    v[2] = __builtin_amdgcn_cvt_f32_fp8(q, 2) * scale;
    v[3] = __builtin_amdgcn_cvt_f32_fp8(q, 3) * scale;
}

// The magnitude a block's scale goes by: at least 1e-30 (a block of zeros keeps a
// finite scale); a NaN stays one, and makes the block's codes NaN.
__device__ inline float scale_top(float top) { return top < 1e-30f ? 1e-30f : top; }

// Four codes, `left` of them there.
__device__ inline void store_codes(unsigned char *to, unsigned q, int left) {
    if (left >= 4) {
        *reinterpret_cast<unsigned *>(to) = q;
    } else {
        for (int e = 0; e < left; ++e) to[e] = (unsigned char)(q >> 8 * e);
    }
}

template <bool EIGHT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwArgs a) {
    const AdamwChunk c = a.chunks[blockIdx.x];
    const AdamwTensor t = a.tensors[c.tensor];
    const void *grad = a.grads[c.tensor];
    const int grad_type = a.grad_type[c.tensor];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = wave; b < kAdamwChunk / kAdamwBlock; b += kThreads / 64) {
        const int64_t at = ((int64_t)c.first + b) * kAdamwBlock + lane * 4;
        if (at - lane * 4 >= t.count) break;
        const int left = (int)(t.count - at < 4 ? (t.count - at > 0 ? t.count - at : 0) : 4);
        const int64_t st = t.state + at;   // a multiple of 4
        float g[4], p[4], m[4], v[4], root[4];
        read_any(grad_type, grad, at, left, g);
        if (a.master) read_typed<float>(a.master, st, left, p);
        else read_any(t.type, t.param, at, left, p);
        if (EIGHT) {
            const unsigned qm = left ? static_cast<const unsigned *>(a.mean)[st / 4] : 0;
            const unsigned qv = left ? static_cast<const unsigned *>(a.square)[st / 4] : 0;
            from_codes(qm, a.mean_scale[st / kAdamwBlock], m);
            from_codes(qv, a.square_scale[st / kAdamwBlock], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = v[e] * v[e];
        } else {
            read_typed<float>(a.mean, st, left, m);
            read_typed<float>(a.square, st, left, v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = m[e] * a.beta1 + g[e] * a.rest1;
            v[e] = v[e] * a.beta2 + (g[e] * g[e]) * a.rest2;
            root[e] = sqrtf(v[e]);
            p[e] = p[e] * a.decay - (m[e] * a.rate) / (root[e] * a.root_scale + a.eps);
        }
        if (a.master) write_typed<float>(a.master, st, left, p);
        write_any(t.type, t.param, at, left, p);
        if (EIGHT) {
            // what lies past the tensor's end takes no part
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e >= left) m[e] = root[e] = 0.f;
            // in units of 448 / top, as a reciprocal and a product
            const float tm = scale_top(wave_top(m)), tr = scale_top(wave_top(root));
            const float im = (1.f / tm) * 448.f, ir = (1.f / tr) * 448.f;
            float qm[4], qr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                qm[e] = m[e] * im;
                qr[e] = root[e] * ir;
                // half of the least code and less would round to 0
                if (root[e] > 0.f && qr[e] <= 0x1p-10f) qr[e] = 0x1p-9f;
            }
            if (left) {
                store_codes(static_cast<unsigned char *>(a.mean) + st, to_codes(qm), left);
                store_codes(static_cast<unsigned char *>(a.square) + st, to_codes(qr), left);
            }
            if (lane == 0) {
                a.mean_scale[st / kAdamwBlock] = tm * (1.f / 448.f);
                a.square_scale[st / kAdamwBlock] = tr * (1.f / 448.f);
            }
        } else {
            write_typed<float>(a.mean, st, left, m);
            write_typed<float>(a.square, st, left, v);
        }
    }
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs &a, bool eight, hipStream_t stream) {
    if (a.nchunks == 0) return hipSuccess;
    if (eight) adamw_kernel<true><<<a.nchunks, kThreads, 0, stream>>>(a);
    else adamw_kernel<false><<<a.nchunks, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace som
