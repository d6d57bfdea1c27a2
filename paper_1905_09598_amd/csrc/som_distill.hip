// A loss from a teacher's top logits and from labels, and its gradient, in one read of
// the logits (the formulas are som_local.h's).  Of a row s of `classes` logits with its
// maximum m, and c = log2(e) / temperature:
//     Z = sum of 2^((s - m) c),    R = the same over the classes that the teacher left out,
//     E = sum of e^(s - m)         (labels only)
// give the loss, and with them the gradient is an exponential or two of each logit again.
// Bound by memory, logits read and gradients written once, and behind that by the
// exponentials: a quarter of the rate of other instructions, two to four a logit.
// A row stays in registers as it was read, 16-byte pieces of it to a lane, of 1 to 64
// lanes or of a workgroup; only rows beyond what a workgroup holds are read twice.  R is
// summed by itself (Z less the teacher's classes would cancel): the teacher's classes are
// marked by bits in LDS, of which a piece of a row takes its own in one read.  Where R is
// next to nothing it is summed once more, from its own classes' maximum (kApart).  All
// gradients are written as if no class were named, and the few that are once more behind a
// barrier.  What a row has beside its logits is read while they are on their way.  16,001
// bf16 rows of 10,000, eight named classes and labels, take 151 us (4.2 TB/s); with the
// named classes tested for on the way, and the rest read when it was needed, 198.  Rows of
// 200,003 are read twice: 512 of them 146 us (instructions 83 of it by count).
#include "som_row.h"

#include <algorithm>
#include <math.h>

namespace som {
namespace {

constexpr float kLog2e = 1.44269504f;

// What the teacher says of a workgroup's rows, in LDS: for each row bits of its classes,
// its entries (a class, or -1 for none, its probability and its logit) and its rest.
inline __host__ __device__ int taught_words(const DistillArgs &a) { return a.words + 3 * a.k + 2; }
struct Taught {
    uint32_t *bits;
    int *index;
    float *p, *logit, *rest;
    __device__ Taught(char *lds, int row, const DistillArgs &a) {
        bits = reinterpret_cast<uint32_t *>(lds) + row * taught_words(a);
        index = reinterpret_cast<int *>(bits + a.words);
        p = reinterpret_cast<float *>(index + a.k);
        logit = p + a.k;
        rest = logit + a.k;   // the rest; 1 where there is a teacher, 0 where not, NaN for NaN
    }
    // The marks of the N classes from `at` on.
    template <int N>
    __device__ uint32_t marks(int at) const {
        const uint32_t *const w = bits + (at >> 5);
        const uint64_t both = (uint64_t)w[1] << 32 | w[0];
        return (uint32_t)(both >> (at & 31)) & ((1u << N) - 1);
    }
};

__device__ inline float wide(const void *p, int32_t type, int64_t i) {
    return type == kF32    ? static_cast<const float *>(p)[i]
           : type == kBF16 ? (float)static_cast<const __bf16 *>(p)[i]
                           : (float)static_cast<const _Float16 *>(p)[i];
}

// The sum over `lanes` neighbours, at most a wave.
__device__ inline float lanes_sum(float v, int lanes) {
    for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor(v, o);
    return v;
}

// The entries of row s, by `lanes` lanes of one wave that cover the row's `lane` 0 ..
// The bits are zeros before.
template <typename T>
__device__ inline void teach(const DistillArgs &a, const Taught &t, const T *s, int64_t row,
                             bool there, int lane, int lanes) {
    float best = -INFINITY, sum = 0.f, rest = a.rest && there ? a.rest[row] : 0.f;
    for (int j = lane; j < a.k; j += lanes) {
        const int64_t at = row * a.k + j;
        int c = there ? a.index[at] : -1;
        const float said = there ? wide(a.teacher, a.teacher_type, at) : 0.f;
        if (c < 0 || c >= a.classes) c = -1;
        const float v = c >= 0 ? said : -INFINITY;
        t.index[j] = c;
        t.p[j] = v;
        t.logit[j] = c >= 0 ? (float)s[c] : 0.f;
        if (a.words && c >= 0) atomicOr(t.bits + (c >> 5), 1u << (c & 31));
        best = fmaxf(best, v);
    }
    for (int o = 1; o < lanes; o <<= 1) best = fmaxf(best, __shfl_xor(best, o));
    const float from = best > -INFINITY ? best : 0.f;   // nothing: e^-inf below is 0
    for (int j = lane; j < a.k; j += lanes) {
        // over the temperature behind the difference: before it fp32 may not hold them
        const float e = expf((t.p[j] - from) / a.temperature);
        t.p[j] = e;
        sum += e;
    }
    sum = lanes_sum(sum, lanes);
    rest = rest <= 0.f || sum == 0.f ? 0.f : rest > 1.f ? 1.f : rest;
    const float by = (1.f - rest) / (sum == 0.f ? 1.f : sum);
    for (int j = lane; j < a.k; j += lanes) t.p[j] *= by;
    if (lane == 0) {
        t.rest[0] = rest;
        t.rest[1] = sum == 0.f ? 0.f : sum / sum;
    }
}

// How labels' exponentials come.  At temperatures of 1, 2 and 4 they are the others', squared
// none, one or two times, off by no more than by themselves: the error of the product in the
// exponent doubles with the exponent either way.  (16,001 bf16 rows of 10,000 at 2: 167 us
// with exponentials of their own, 156 so.)
enum : int { kNoLabels = 0, kOwn = 1, kSame = 2, kSquared = 3, kTwice = 4 };

// 2^((v - top) c) of N logits and, with labels, e^(v - top).
template <int HARD, int N>
__device__ inline void powers(const float (&v)[N], float top, float c, float (&soft)[N],
                              float (&hard)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float u = v[e] - top;
        soft[e] = __builtin_amdgcn_exp2f(u * c);
        if (HARD == kOwn) hard[e] = __builtin_amdgcn_exp2f(u * kLog2e);
        if (HARD >= kSame) hard[e] = soft[e];
        if (HARD >= kSquared) hard[e] *= hard[e];
        if (HARD >= kTwice) hard[e] *= hard[e];
    }
}

// What a row has beside its teacher, read while its logits are on their way.
struct Beside {
    float scale, logit;   // of the gradient; the label's
    int at;               // the label's class, or -1
    template <int HARD, typename T>
    __device__ static Beside of(const DistillArgs &a, const T *s, int64_t row, bool there) {
        Beside b;
        b.scale = a.dloss && there ? a.scale * a.dloss[row] : a.scale;
        b.at = HARD && there ? a.label[row] : -1;
        if (b.at >= a.classes || b.at < 0) b.at = -1;
        b.logit = b.at >= 0 ? (float)s[b.at] : 0.f;
        return b;
    }
};

// Of rows whose classes that the teacher left out have less than this of the sum, R and its
// exponentials are taken from those classes' own maximum: counted from the row's they would
// be 0 from 87 temperatures below it on, where R's logarithm and their shares of the rest
// are numbers like others.  (What 2^-60 is next to: an element left out at 2^-126 is 2^-66
// of it.)
constexpr float kApart = 0x1p-60f;

// What a row's sums give.
struct Factors {
    float z, r, e;                  // the sums
    float t;                        // of the teacher's classes: z - r
    float top, chosen, other, one;  // m; factors of 2^((s - m) c) and of e^(s - m)
    float given;                    // of the teacher's probability
    float label;                    // of the label's class
    bool shut;                      // a row without an open class
    bool apart;                     // r counts from `lead`, the maximum of those classes,
    float lead, left;               // and `left` is the factor of their 2^((s - lead) c)
    // Whether it does; alike for all lanes of a row.
    __device__ static bool is_apart(const DistillArgs &a, const Taught &t, const float (&sums)[3]) {
        return a.words && t.rest[0] > 0.f && sums[1] < kApart;
    }
    // Takes r from there: far, unless none of those classes is open.
    __device__ void part(const Taught &t, float from, float far) {
        if (!(from > -INFINITY)) return;
        apart = true, lead = from, r = far;
        if (given != 0.f) other = chosen, left = given * t.rest[0] / far;
    }
    template <int HARD>
    __device__ static Factors of(const DistillArgs &a, const Taught &t, const Beside &b, float top,
                                 const float (&sums)[3]) {
        Factors f;
        const float z = sums[0] + sums[1], r = sums[1], e = sums[2];
        f.z = z, f.r = r, f.e = e, f.t = sums[0], f.top = top;
        f.apart = false, f.lead = f.left = 0.f;
        f.shut = z == 0.f;
        const float soft = b.scale * a.mix * a.temperature, hard = b.scale * (1.f - a.mix);
        // a logit that is none: all of the row is none, also without a part of its own
        f.chosen = f.other = z == z ? 0.f : z;
        f.given = f.one = f.label = 0.f;
        if (f.shut) return f;
        if (a.k && a.mix != 0.f && !(t.rest[1] == 0.f)) {
            f.given = soft * t.rest[1];
            f.chosen = f.given / z;
            f.other = f.chosen;
            // the classes that the teacher left out, whose sum is to be its rest: from the
            // smaller of the two parts of z, so that what is left of 1 keeps its bits
            const float rest = t.rest[0];
            if (rest != 0.f && r == 0.f) f.other = 0.f;
            else if (rest != 0.f)
                f.other = f.chosen * (f.t < r ? ((1.f - rest) - f.t / z) * (z / r) : 1.f - rest * (z / r));
        }
        if (HARD && b.at >= 0) f.one = hard / e, f.label = hard;
        return f;
    }
};

// The row's loss, by `lanes` lanes of one wave.
template <int HARD>
__device__ inline float loss_of(const DistillArgs &a, const Taught &t, const Factors &f, const Beside &b,
                                int lane, int lanes) {
    if (f.shut) return 0.f;
    if (f.z != f.z) return f.z;
    float soft = 0.f, away = 0.f, all = 0.f;   // of logarithms; of distances below the maximum
    // half of a logit's distance from the maximum, and not over the temperature: the whole,
    // and what a low temperature makes of it, may pass fp32's range where the loss does not
    const auto half_below = [&](float v) { return 0.5f * v - 0.5f * f.top; };
    if (a.k && a.mix != 0.f) {
        const float log_z = logf(f.z);
        for (int j = lane; j < a.k; j += lanes) {
            const float p = t.p[j];
            if (t.index[j] < 0 || p == 0.f) continue;
            soft = fmaf(p, logf(p) + log_z, soft);
            away = fmaf(-p, half_below(t.logit[j]), away);
        }
        soft = lanes_sum(soft, lanes);
        away = lanes_sum(away, lanes);
        const float rest = t.rest[0];
        if (rest != 0.f) {   // next to 1 a share's logarithm comes from the other share
            const float share = !f.apart && f.t < f.r ? log1pf(-f.t / f.z) : logf(f.r / f.z);
            soft = fmaf(rest, logf(rest) - share, soft);
            if (f.apart) away = fmaf(-rest, half_below(f.lead), away);
        }
        if (t.rest[1] != 1.f) soft = t.rest[1];   // 0 or NaN
        const float by = a.mix * a.temperature;
        all = fmaf(2.f * by, away, by * a.temperature * soft);
    }
    if (HARD && b.at >= 0) {
        const float part = 1.f - a.mix;
        all += fmaf(part, logf(f.e), -2.f * (part * half_below(b.logit)));
    }
    return all;
}

// The gradient of N neighbouring logits v, as of classes that neither the teacher nor the
// label names.
template <int HARD, int N>
__device__ inline void slopes(const Factors &f, float c, float (&v)[N]) {
    float soft[N], hard[N];
    powers<HARD>(v, f.top, c, soft, hard);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        v[e] = f.other * soft[e];
        if (HARD) v[e] = fmaf(f.one, hard[e], v[e]);
    }
}

// Rows whose R counts from its own classes' maximum, by all of a row's lanes: seldom, so they
// are read again, a class at a time, for which the registers that hold a row need not make
// room.  The sum from the maximum `lead` of the classes that the teacher left out.
template <bool WIDE, typename T>
__device__ inline float apart_sum(const DistillArgs &a, const Taught &t, const T *s, int lane, int lanes,
                                  float c, float *part, int &turn, float *lead) {
    float most[1] = {-INFINITY}, sum[1] = {0.f};
#pragma unroll 1
    for (int at = lane; at < a.classes; at += lanes)
        if (!t.template marks<1>(at)) most[0] = fmaxf(most[0], (float)s[at]);
    row_max<WIDE>(most, lanes, part, turn);
#pragma unroll 1
    for (int at = lane; at < a.classes; at += lanes)
        if (!t.template marks<1>(at)) sum[0] += __builtin_amdgcn_exp2f(((float)s[at] - most[0]) * c);
    row_sum<WIDE>(sum, lanes, part, turn);
    *lead = most[0];
    return sum[0];
}
// The gradient, as slopes gives it.
template <int HARD, typename T>
__device__ inline void apart_slopes(const DistillArgs &a, const Factors &f, const T *s, T *to, int lane,
                                    int lanes, float c) {
#pragma unroll 1
    for (int at = lane; at < a.classes; at += lanes) {
        const float logit = (float)s[at];
        float v[1] = {logit};
        slopes<HARD>(f, c, v);
        if (f.apart) v[0] = fmaf(-f.left, __builtin_amdgcn_exp2f((logit - f.lead) * c), v[0]);
        to[at] = (T)v[0];
    }
}

// The named classes' gradients, written over those, by `lanes` lanes of one wave.  All of
// a row's other writes come before (a barrier); classes that are named more than once
// are written by several lanes, all alike.
template <typename T, int HARD>
__device__ inline void named(const DistillArgs &a, const Taught &t, const Factors &f, const Beside &b,
                             T *to, float c, int lane, int lanes) {
    for (int j = lane; j < a.k + (HARD ? 1 : 0); j += lanes) {
        const int at = j < a.k ? t.index[j] : b.at;
        if (at < 0) continue;
        float p = 0.f;
        bool taught = false;
        for (int i = 0; i < a.k; ++i) {
            const bool same = t.index[i] == at;
            p += same ? t.p[i] : 0.f;
            taught = taught || same;
        }
        const float logit[1] = {j < a.k ? t.logit[j] : b.logit};
        float soft[1], hard[1];
        powers<HARD>(logit, f.top, c, soft, hard);
        float v = (taught ? f.chosen : f.other) * soft[0];
        if (taught) v -= f.given * p;
        else if (f.apart) v = fmaf(-f.left, __builtin_amdgcn_exp2f((logit[0] - f.lead) * c), v);
        if (HARD) v = fmaf(f.one, hard[0], v);
        if (HARD && at == b.at) v -= f.label;
        to[at] = (T)v;
    }
}

template <typename T, int P, bool WIDE, int HARD>
__global__ __launch_bounds__(1024) void distill_kernel(DistillArgs a) {
    constexpr int N = 16 / sizeof(T);
    extern __shared__ char lds[];
    __shared__ __align__(16) float part[WIDE ? kPart : 1];
    int turn = 0;
    const Part<WIDE, P, N> me(a.lanes, a.classes);
    const int64_t row = (int64_t)blockIdx.x * me.rows + me.row;
    const bool there = row < a.n;
    const T *const s = static_cast<const T *>(a.logits) + row * a.lds;
    Piece<T, N> x[P];
#pragma unroll
    for (int p = 0; p < P; ++p) me.template read<T>(s, 0, p, there, x[p]);
    const Beside beside = Beside::of<HARD>(a, s, row, there);
    const Taught t(lds, me.row, a);
    const bool first = !WIDE || threadIdx.x < 64;      // those that deal with entries
    const int lanes = WIDE ? 64 : a.lanes;
    if (a.k) {
        for (int w = me.lane; w < a.words; w += a.lanes) t.bits[w] = 0;
        __syncthreads();
        if (first) teach(a, t, s, row, there, me.lane, lanes);
        if (!WIDE) __syncthreads();                    // otherwise the maximum's
    }
    // -infinity where a piece is not this lane's
    const auto values = [&](int p, float (&v)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)x[p].v[e];
        if (me.skip[p] > 0) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = e < me.skip[p] ? -INFINITY : v[e];
        }
    };
    float top[1] = {-INFINITY};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float v[N];
        values(p, v);
#pragma unroll
        for (int e = 0; e < N; ++e) top[0] = fmaxf(top[0], v[e]);
    }
    row_max<WIDE>(top, a.lanes, part, turn);
    keep_raw<T, P>(x);
    const float from = top[0] > -INFINITY ? top[0] : 0.f, c = kLog2e / a.temperature;
    // the teacher's classes, the others, and all with the exponentials of labels
    float sums[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float v[N];
        values(p, v);
        const uint32_t marks = a.words && me.mine(p) ? t.template marks<N>(me.at[p]) : 0u;
        float soft[N], hard[N];
        powers<HARD>(v, from, c, soft, hard);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            v[e] = soft[e];
            if (HARD) sums[2] += hard[e];
        }
        if (marks) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sums[0] += marks >> e & 1 ? v[e] : 0.f;
                v[e] = marks >> e & 1 ? 0.f : v[e];
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sums[1] += v[e];
        // one piece after the other: together, without labels' exponentials between, they take
        // 72 registers and not 58 (16,001 bf16 rows of 10,000: 151 us and not 144)
        if (!HARD) asm volatile("" : "+v"(sums[1]));
    }
    row_sum<WIDE>(sums, a.lanes, part, turn);
    keep_raw<T, P>(x);
    T *const to = static_cast<T *>(a.dlogits) + row * a.classes;
    Factors f = Factors::of<HARD>(a, t, beside, from, sums);
    bool apart = Factors::is_apart(a, t, sums);
    if (WIDE) apart = __builtin_amdgcn_readfirstlane(apart);   // as it is for all
    if (!there) return;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!a.dlogits || apart || !me.mine(p)) continue;
        float v[N];
        Piece<T, N> out;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)x[p].v[e];
        slopes<HARD>(f, c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) out.v[e] = (T)v[e];
        out.write(to + me.at[p], N);
    }
    if (apart) {   // here, where the row's registers are free
        float lead;
        const float far = apart_sum<WIDE>(a, t, s, me.lane, a.lanes, c, part, turn, &lead);
        f.part(t, lead, far);
        if (a.dlogits) apart_slopes<HARD>(a, f, s, to, me.lane, a.lanes, c);
    }
    if (WIDE) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");   // one wave
    if (!first) return;
    if (a.dlogits) named<T, HARD>(a, t, f, beside, to, c, me.lane, lanes);
    if (a.loss) {
        const float loss = loss_of<HARD>(a, t, f, beside, me.lane, lanes);
        if (me.lane == 0) a.loss[row] = loss;
    }
}

// Rows that a workgroup does not hold, and rows shorter than a piece: read twice, with
// the maximum and the sums of what a lane has seen so far in the first pass.
template <typename T, int HARD>
__global__ __launch_bounds__(1024) void distill_long_kernel(DistillArgs a) {
    constexpr int N = 16 / sizeof(T), kAhead = 4;
    extern __shared__ char lds[];
    __shared__ __align__(16) float part[kPart];
    int turn = 0;
    const int64_t row = blockIdx.x;
    const T *const s = static_cast<const T *>(a.logits) + row * a.lds;
    const Beside beside = Beside::of<HARD>(a, s, row, true);
    const Taught t(lds, 0, a);
    const bool first = threadIdx.x < 64;
    if (a.k) {
        for (int w = threadIdx.x; w < a.words; w += blockDim.x) t.bits[w] = 0;
        __syncthreads();
        if (first) teach(a, t, s, row, true, threadIdx.x, 64);
        __syncthreads();
    }
    const float c = kLog2e / a.temperature;
    const int stride = blockDim.x * N;
    float top[1] = {-INFINITY}, from = 0.f, sums[3] = {0.f, 0.f, 0.f};
    // kAhead pieces of this lane are read together, from class `at` on
    const auto read = [&](int at, Piece<T, N> (&x)[kAhead]) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int left = a.classes - (at + q * stride);
            x[q].read(s + at + q * stride, left < 0 ? 0 : left < N ? left : N);
        }
    };
    for (int first_at = threadIdx.x * N; first_at < a.classes; first_at += kAhead * stride) {
        Piece<T, N> x[kAhead];
        read(first_at, x);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int at = first_at + q * stride, left = a.classes - at;
            if (left <= 0) break;
            float v[N], most = -INFINITY;
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (float)x[q].v[e];
            if (left < N) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = e < left ? v[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, v[e]);
            if (most > top[0]) {
                const float u = top[0] > -INFINITY ? from - most : 0.f;   // sums of nothing stay 0
                sums[0] *= __builtin_amdgcn_exp2f(u * c);
                sums[1] *= __builtin_amdgcn_exp2f(u * c);
                if (HARD) sums[2] *= __builtin_amdgcn_exp2f(u * kLog2e);
                top[0] = from = most;
            }
            const uint32_t marks = a.words ? t.template marks<N>(at) : 0u;
            float soft[N], hard[N];
            powers<HARD>(v, from, c, soft, hard);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[e] = soft[e];
                if (HARD) sums[2] += hard[e];
            }
            if (marks) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    sums[0] += marks >> e & 1 ? v[e] : 0.f;
                    v[e] = marks >> e & 1 ? 0.f : v[e];
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) sums[1] += v[e];
        }
    }
    const float mine = top[0];
    row_max<true>(top, 0, part, turn);
    const float all = top[0] > -INFINITY ? top[0] : 0.f;
    if (mine > -INFINITY) {
        sums[0] *= __builtin_amdgcn_exp2f((mine - all) * c);
        sums[1] *= __builtin_amdgcn_exp2f((mine - all) * c);
        if (HARD) sums[2] *= __builtin_amdgcn_exp2f((mine - all) * kLog2e);
    }
    row_sum<true>(sums, 0, part, turn);
    Factors f = Factors::of<HARD>(a, t, beside, all, sums);
    if (Factors::is_apart(a, t, sums)) {
        float lead;
        const float far = apart_sum<true>(a, t, s, threadIdx.x, blockDim.x, c, part, turn, &lead);
        f.part(t, lead, far);
    }
    if (a.loss && first) {
        const float loss = loss_of<HARD>(a, t, f, beside, threadIdx.x, 64);
        if (threadIdx.x == 0) a.loss[row] = loss;
    }
    if (!a.dlogits) return;
    T *const to = static_cast<T *>(a.dlogits) + row * a.classes;
    if (f.apart) apart_slopes<HARD>(a, f, s, to, threadIdx.x, blockDim.x, c);
    for (int first_at = threadIdx.x * N; !f.apart && first_at < a.classes; first_at += kAhead * stride) {
        Piece<T, N> x[kAhead];
        read(first_at, x);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int at = first_at + q * stride, left = a.classes - at;
            if (left <= 0) break;
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (float)x[q].v[e];
            slopes<HARD>(f, c, v);
#pragma unroll
            for (int e = 0; e < N; ++e) x[q].v[e] = (T)v[e];
            x[q].write(to + at, left < N ? left : N);
        }
    }
    __syncthreads();
    if (first) named<T, HARD>(a, t, f, beside, to, c, threadIdx.x, 64);
}

// Pieces that a lane holds: 1, 2 or 4 of a row that a wave or less takes, 4 or 8 of one that
// a workgroup takes (16 are more than the registers of 1024 threads).  Short rows wait for
// their reads and reductions, not for memory: of many rows a lane takes more pieces, so that
// a wave has more rows under way (60,000 bf16 rows of 400: one piece 71 us, four 36; of 1000
// two 88, four 63), of few rows one, so that they are on more compute units.  Rows of more
// than 128 pieces go to a workgroup (60,000 of 1030: 91 us, to the lanes of a wave 104).
constexpr int kNarrowPieces = 4, kWidePieces = 8;
constexpr int64_t kManyWaves = 4096;   // 16 to a compute unit

Shape distill_shape(const DistillArgs &a) {
    Shape s = shape_of(a.type, a.classes, 2, kWidePieces, 64);
    if (s.held && s.wide) {
        const int n = 16 / type_size(a.type), pieces = (a.classes + n - 1) / n;
        s.pieces = pieces > 1024 * 4 ? 8 : 4;
        s.threads = s.lanes = (pieces + 64 * s.pieces - 1) / (64 * s.pieces) * 64;
    } else if (s.held) {
        while (s.pieces < kNarrowPieces && s.lanes > 1 && a.n * s.lanes > kManyWaves * 64)
            s.pieces *= 2, s.lanes /= 2;
    }
    return s;
}

template <typename T, int P, bool WIDE, int HARD>
hipError_t launch_held(const DistillArgs &a, const Shape &s, unsigned groups, unsigned lds,
                       hipStream_t stream) {
    distill_kernel<T, P, WIDE, HARD><<<groups, s.threads, lds, stream>>>(a);
    return hipGetLastError();
}

template <typename T, int HARD>
hipError_t launch_typed(const DistillArgs &a, const Shape &s, unsigned groups, unsigned lds,
                        hipStream_t stream) {
    if (!s.held) {
        const auto kernel = distill_long_kernel<T, HARD>;
        if (lds > 60 * 1024) {
            const hipError_t e =
                hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        kernel<<<groups, s.threads, lds, stream>>>(a);
        return hipGetLastError();
    }
    if (!s.wide) {
        return s.pieces == 1   ? launch_held<T, 1, false, HARD>(a, s, groups, lds, stream)
               : s.pieces == 2 ? launch_held<T, 2, false, HARD>(a, s, groups, lds, stream)
                               : launch_held<T, 4, false, HARD>(a, s, groups, lds, stream);
    }
    return s.pieces == 4 ? launch_held<T, 4, true, HARD>(a, s, groups, lds, stream)
                         : launch_held<T, 8, true, HARD>(a, s, groups, lds, stream);
}

template <typename T>
hipError_t launch_labels(const DistillArgs &a, int hard, const Shape &s, unsigned groups, unsigned lds,
                         hipStream_t stream) {
    switch (hard) {
        case kNoLabels: return launch_typed<T, kNoLabels>(a, s, groups, lds, stream);
        case kOwn: return launch_typed<T, kOwn>(a, s, groups, lds, stream);
        case kSame: return launch_typed<T, kSame>(a, s, groups, lds, stream);
        case kSquared: return launch_typed<T, kSquared>(a, s, groups, lds, stream);
        default: return launch_typed<T, kTwice>(a, s, groups, lds, stream);
    }
}

}  // namespace

hipError_t launch_distill(const DistillArgs &args, hipStream_t stream) {
    const Shape s = distill_shape(args);
    const int rows = s.held && !s.wide ? s.threads / s.lanes : 1;
    DistillArgs a = args;
    a.lanes = s.lanes;
    a.words = a.k && a.rest ? (a.classes + 31) / 32 + 1 : 0;   // its sum leaves classes out
    const unsigned lds = (unsigned)rows * taught_words(a) * 4;
    const int size = type_size(a.type);
    const int hard = !a.label || a.mix == 1.f   ? kNoLabels
                     : a.temperature == 1.f ? kSame
                     : a.temperature == 2.f ? kSquared
                     : a.temperature == 4.f ? kTwice
                                            : kOwn;
    // as many rows at a time as a grid holds
    const int64_t most = (int64_t)(UINT32_MAX / 1024) * rows;
    for (int64_t r = 0; r < args.n; r += most) {
        a.n = std::min(most, args.n - r);
        const unsigned groups = (unsigned)((a.n + rows - 1) / rows);
        hipError_t e;
        switch (a.type) {
            case kF32: e = launch_labels<float>(a, hard, s, groups, lds, stream); break;
            case kBF16: e = launch_labels<__bf16>(a, hard, s, groups, lds, stream); break;
            default: e = launch_labels<_Float16>(a, hard, s, groups, lds, stream);
        }
        if (e != hipSuccess) return e;
        a.logits = static_cast<const char *>(a.logits) + a.n * a.lds * size;
        if (a.index) a.index += a.n * a.k;
        if (a.teacher) a.teacher = static_cast<const char *>(a.teacher) + a.n * a.k * type_size(a.teacher_type);
        if (a.rest) a.rest += a.n;
        if (a.label) a.label += a.n;
        if (a.dloss) a.dloss += a.n;
        if (a.loss) a.loss += a.n;
        if (a.dlogits) a.dlogits = static_cast<char *>(a.dlogits) + a.n * a.classes * size;
    }
    return hipSuccess;
}

}  // namespace som
