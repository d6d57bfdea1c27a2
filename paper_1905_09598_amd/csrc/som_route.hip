// Routing: which experts a document goes to, with which weights, and the
// documents in the order of their experts.
//
// route: a row of scores lies in the registers of 16 lanes or of a wave, V
// neighbours to a lane, so that the lowest lane and element of equal values is the
// lowest expert; rows of more than 2048 experts lie in LDS, one to a workgroup.
// The k choices are k maxima over the row, of whole numbers in the values' order:
// one per lane, joined across the lanes by rotations; only the lane that won
// takes its element out.  Bound by these instructions, not by the read of the scores
// (65,536 bf16 rows of 256 experts in 8 groups, 8 choices of sigmoids with a bias: 42 us,
// of which the read would take 7; 20,000 fp32 rows of 400, 4 choices: 21 us).
// Sixteen lanes hold a row where they can: the steps across lanes are shared by the four
// rows of a wave (the same rows of 256 a wave each 80 us, of 64 experts 17 and 22 us).
#include "som_local_internal.h"

#include <float.h>
#include <math.h>

namespace som {
namespace {

constexpr int kRouteThreads = 256;

template <int LANES, typename F>
__device__ inline float across(float v, F join) {
    // rotations within rows of 16 lanes, then across the rows
    v = join(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xf, 0xf, false)));
    v = join(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124, 0xf, 0xf, false)));
    v = join(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x122, 0xf, 0xf, false)));
    v = join(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x121, 0xf, 0xf, false)));
    if (LANES == 64) {
        v = join(v, __shfl_xor(v, 16));
        v = join(v, __shfl_xor(v, 32));
    }
    return v;
}
template <int LANES>
__device__ inline float across_max(float v) {
    return across<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
// In the same order for every lane: the sum is the same in all of them.
template <int LANES>
__device__ inline float across_sum(float v) {
    return across<LANES>(v, [](float a, float b) { return a + b; });
}

// The lanes of this lane's row of LANES for which `is` holds, the row's first
// lane in bit 0.
template <int LANES>
__device__ inline unsigned long long row_ballot(bool is) {
    const unsigned long long all = __ballot(is);
    return LANES == 64 ? all : all >> (threadIdx.x & 48) & 0xffff;
}

// 1 / (1 + e^-s) in the roundings of its three operations.  The division: the
// hardware's reciprocal is within one unit in the last place, and a step of
// Newton's in fused operations rounds it correctly (Markstein), in a third of the
// instructions.  Beyond 2^126, where the reciprocal would be denormal, the
// divisor is scaled; infinity gives 0.
constexpr float kNear = 80.f;   // scores from -80 on are not that far
template <bool NEAR = false>
__device__ inline float sigmoid(float s) {
    const float d = 1.f + expf(-s);
    const bool far = !NEAR && d >= 0x1p126f;
    const float b = far ? d * 0x1p-64f : d;
    const float r = __builtin_amdgcn_rcpf(b);
    const float q = fmaf(fmaf(-b, r, 1.f), r, r);
    return far ? (d < INFINITY ? q * 0x1p-64f : 0.f) : q;
}

// Whole numbers in the order of the floats (equal zeros alike), the least for
// -infinity; those of NaN are never looked at.
__device__ inline int key_of(float v) {
    const int b = __float_as_int(v + 0.f);
    return b ^ (b >> 31 & 0x7fffffff);
}
constexpr int kClosed = (int)(0xff800000u ^ 0x7fffffffu);

template <int LANES>
__device__ inline int across_max_key(int v) {
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x124, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x122, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x121, 0xf, 0xf, false));
    if (LANES == 64) {
        v = max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
                max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
    }
    return v;
}

// Whether this is the first lane of its row for which `is` holds.
template <int LANES>
__device__ inline bool first_of_row(bool is, int lane) {
    const unsigned long long all = __ballot(is);
    if (LANES == 64) return is && (all & ((1ull << lane) - 1)) == 0;
    const unsigned half = (unsigned)(threadIdx.x & 32 ? all >> 32 : all) >> (threadIdx.x & 16);
    return is && (half & ((1u << lane) - 1)) == 0;
}

// V neighbouring values of a row from element e0 on, `fill` past its end.
template <typename T, int V>
__device__ inline void read_row(const T *s, int e0, int experts, float fill, float (&x)[V]) {
    typedef T Vec __attribute__((ext_vector_type(V)));
    if (e0 + V <= experts) {
        Vec q;
        __builtin_memcpy(&q, __builtin_assume_aligned(s + e0, sizeof(T)), sizeof(T) * V);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = (float)q[v];
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = e0 + v < experts ? (float)s[e0 + v] : fill;
    }
}
template <typename T, int V>
__device__ inline void write_row(T *s, int e0, int experts, const float (&x)[V]) {
    typedef T Vec __attribute__((ext_vector_type(V)));
    if (e0 + V <= experts) {
        Vec q;
#pragma unroll
        for (int v = 0; v < V; ++v) q[v] = (T)x[v];
        __builtin_memcpy(__builtin_assume_aligned(s + e0, sizeof(T)), &q, sizeof(T) * V);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (e0 + v < experts) s[e0 + v] = (T)x[v];
    }
}

// The value that the choice goes by; -infinity: closed.  p: the sigmoid of the score,
// or the score itself.
__device__ inline float choice_value(float s, float p, float bias) {
    return s > -INFINITY ? fmaxf(p + bias, -INFINITY) : -INFINITY;   // NaN: -infinity
}

// A group's value from its two largest; one with an open expert is open, also where
// the sum of two lowest values passes fp32's range.
__device__ inline float group_of(float best, float next, int count) {
    return count == 2 && next > -INFINITY ? fmaxf(best + next, -FLT_MAX) : best;
}

// Whether a score makes its whole row invalid.
__device__ inline bool spoils(float s, bool softmax) {
    return s != s || (softmax && s == INFINITY);
}

// The groups that stay, as bits.  Lane g << shift holds group g's value.
template <int LANES>
__device__ inline unsigned long long groups_that_stay(float value, int lane, int shift, int groups,
                                                      int top) {
    const int mine = lane >> shift;
    int before = 0;
    for (int h = 0; h < groups; ++h) {
        const float other = __shfl(value, h << shift, LANES);
        before += other > value || (other == value && h < mine) ? 1 : 0;
    }
    const bool stays = (lane & ((1 << shift) - 1)) == 0 && mine < groups && before < top &&
                       value > -INFINITY;
    const unsigned long long lanes = row_ballot<LANES>(stays);
    if (shift == 0) return lanes;
    unsigned long long bits = 0;
    for (int h = 0; h < groups; ++h) bits |= (lanes >> (h << shift) & 1) << h;
    return bits;
}

// A row's weights from its choices: lane j holds choice j (index at, -1 for none).
// `low`, `total`: the row's largest score and sum of e^(s - low) (softmax that is
// not renormalised).
template <typename T, int LANES>
__device__ inline void write_choices(const RouteArgs &a, int64_t row, int lane, int at, bool bad,
                                     float low, float total) {
    const T *s = static_cast<const T *>(a.scores) + row * a.lds;
    const bool here = lane < a.k && at >= 0;
    const float score = here ? (float)s[at] : -INFINITY;
    float w = 0.f;
    if (a.softmax) {
        if (a.renormalise) {
            float top = across_max<LANES>(score);
            top = top > -INFINITY ? top : 0.f;
            const float e = here ? expf(score - top) : 0.f;
            const float sum = across_sum<LANES>(e);
            w = sum > 0.f ? e / sum : 0.f;
        } else if (here) {
            w = expf(score - low) / total;
        }
    } else {
        w = here ? sigmoid(score) : 0.f;
        if (a.renormalise) {
            const float sum = across_sum<LANES>(w);
            w = sum > 0.f ? w / sum : 0.f;
        }
    }
    if (lane < a.k) {
        a.index[row * a.k + lane] = bad ? -1 : at;
        a.weight[row * a.k + lane] = bad ? NAN : w * a.scale;
    }
}

// The slots of a workgroup's rows in the order of their experts, where these are
// all the slots (up to kSortSlots): a slot's row is the number of slots that come
// before it.  expert: their experts, in LDS.
constexpr int kSortSlots = 64;
__device__ inline void sort_few(const DispatchArgs &a, const int *expert) {
    const int slots = (int)a.slots, t = threadIdx.x;
    if (t < slots) {
        const int e = expert[t];
        int before = 0, there = 0;
        for (int s = 0; s < slots; ++s) {
            const int o = expert[s];
            there += o >= 0 ? 1 : 0;
            before += o >= 0 && (o < e || (o == e && s < t)) ? 1 : 0;
        }
        a.place[t] = e >= 0 ? before : -1;
        if (e >= 0) a.order[before] = t;
        if (t >= there) a.order[t] = -1;
    }
    for (int e = t; e <= a.experts; e += kRouteThreads) {
        int below = 0;
        for (int s = 0; s < slots; ++s) below += expert[s] >= 0 && expert[s] < e ? 1 : 0;
        a.offsets[e] = below;
    }
}

// LANES lanes a row, V experts a lane.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs a, DispatchArgs sort) {
    constexpr int kRows = kRouteThreads / LANES;
    extern __shared__ float shared[];  // with groups that lanes do not hold whole: the values
    __shared__ int chosen[kRows][LANES];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t row = (int64_t)blockIdx.x * kRows + slot;
    const bool there = row < a.n;
    const T *s = static_cast<const T *>(a.scores) + (there ? row : a.n - 1) * a.lds;
    const int e0 = lane * V;
    float x[V];
    read_row<T, V>(s, e0, a.experts, -INFINITY, x);
    bool spoilt = false;
#pragma unroll
    for (int v = 0; v < V; ++v) spoilt |= spoils(x[v], a.softmax);
    const bool bad = row_ballot<LANES>(spoilt) != 0;

    float low = -INFINITY, total = 1.f;
    if (a.softmax && !a.renormalise) {
#pragma unroll
        for (int v = 0; v < V; ++v) low = fmaxf(low, x[v]);
        low = across_max<LANES>(low);
        low = low > -INFINITY ? low : 0.f;
        total = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) total += expf(x[v] - low);
        total = across_sum<LANES>(total);
        total = total > 0.f ? total : 1.f;
    }
    float bias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = 0.f;
    if (a.bias) read_row<float, V>(a.bias, e0, a.experts, 0.f, bias);
    if (a.softmax) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = choice_value(x[v], x[v], bias[v]);
    } else {
        float least = x[0];
#pragma unroll
        for (int v = 1; v < V; ++v) least = fminf(least, x[v]);
        if (__all(least >= -kNear || e0 >= a.experts)) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = choice_value(x[v], sigmoid<true>(x[v]), bias[v]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = choice_value(x[v], sigmoid(x[v]), bias[v]);
        }
    }

    if (a.groups > 1) {
        const int per = a.experts / a.groups, lanes = per / V;
        float best = -INFINITY, next = -INFINITY;
        int shift = 0;
        const bool whole = per % V == 0 && (lanes & (lanes - 1)) == 0;   // lanes, a power of two
        if (whole) {
            shift = 31 - __clz(lanes);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                next = __builtin_amdgcn_fmed3f(best, next, x[v]);   // next <= best
                best = fmaxf(best, x[v]);
            }
            for (int o = 1; o < lanes; o <<= 1) {
                const float b = __shfl_xor(best, o), n = __shfl_xor(next, o);
                next = fmaxf(fmaxf(next, n), fminf(best, b));
                best = fmaxf(best, b);
            }
        } else {
            float *mine = shared + slot * (a.experts + 1);
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (e0 + v < a.experts) mine[e0 + v] = x[v];
            __syncthreads();
            if (lane < a.groups) {   // groups <= LANES
#pragma unroll 4
                for (int e = 0; e < per; ++e) {
                    const float v = mine[lane * per + e];
                    next = fmaxf(next, fminf(best, v));
                    best = fmaxf(best, v);
                }
            }
        }
        const float value = group_of(best, next, a.group_best);
        const unsigned long long stay =
            groups_that_stay<LANES>(value, lane, shift, a.groups, a.top_groups);
        if (whole) {
            const bool stays = stay >> (lane >> shift) & 1;
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = stays ? x[v] : -INFINITY;
        } else {
            int left = per - e0 % per;
            unsigned long long bits = e0 < a.experts ? stay >> e0 / per : 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!(bits & 1)) x[v] = -INFINITY;
                if (--left == 0) bits >>= 1, left = per;
            }
        }
    }

    int key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = key_of(x[v]);
    for (int j = 0; j < a.k; ++j) {
        int best = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = max(best, key[v]);
        const int top = across_max_key<LANES>(best);
        // the first lane that holds it, and its first element
        const bool won = first_of_row<LANES>(best == top, lane);
        int at = 0;
        bool seen = !won;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const bool is = key[v] == top && !seen;
            seen |= is;
            at = is ? v : at;
            key[v] = is ? kClosed : key[v];
        }
        if (won) chosen[slot][j] = top > kClosed ? e0 + at : -1;
    }
    // a row's lanes are in one wave
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int at = lane < a.k ? chosen[slot][lane] : -1;
    if (there) write_choices<T, LANES>(a, row, lane, at, bad, low, total);
    if (sort.offsets) {   // one workgroup
        int *expert = &chosen[0][0];
        __syncthreads();
        if (there && lane < a.k && row * a.k + lane < kSortSlots)
            expert[row * a.k + lane] = bad ? -1 : at;
        __syncthreads();
        sort_few(sort, expert);
    }
}

// One row a workgroup of 256 threads, its values in LDS; thread t looks after
// experts t, t + 256, ...
template <typename T>
__global__ __launch_bounds__(kRouteThreads) void route_long_kernel(RouteArgs a) {
    extern __shared__ float pick[];    // experts values
    __shared__ float part[4];
    __shared__ int where[4];
    __shared__ float group_value[kMaxGroups];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t row = blockIdx.x;
    const T *s = static_cast<const T *>(a.scores) + row * a.lds;
    bool spoilt = false;
    float low = -INFINITY;
    for (int e = t; e < a.experts; e += kRouteThreads) {
        const float x = (float)s[e];
        spoilt |= spoils(x, a.softmax);
        low = fmaxf(low, x);
        pick[e] = choice_value(x, a.softmax ? x : sigmoid(x), a.bias ? a.bias[e] : 0.f);
    }
    const bool bad = __syncthreads_or(spoilt);
    float total = 1.f;
    if (a.softmax && !a.renormalise) {
        low = across_max<64>(low);
        if (lane == 0) part[wave] = low;
        __syncthreads();
        low = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        low = low > -INFINITY ? low : 0.f;
        __syncthreads();
        total = 0.f;
        for (int e = t; e < a.experts; e += kRouteThreads) total += expf((float)s[e] - low);
        total = across_sum<64>(total);
        if (lane == 0) part[wave] = total;
        __syncthreads();
        total = (part[0] + part[1]) + (part[2] + part[3]);
        total = total > 0.f ? total : 1.f;
        __syncthreads();
    }
    if (a.groups > 1) {
        const int per = a.experts / a.groups;
        for (int g = wave; g < a.groups; g += 4) {
            float best = -INFINITY, next = -INFINITY;
            for (int e = lane; e < per; e += 64) {
                const float v = pick[g * per + e];
                next = fmaxf(next, fminf(best, v));
                best = fmaxf(best, v);
            }
            for (int o = 1; o < 64; o <<= 1) {
                const float b = __shfl_xor(best, o), n = __shfl_xor(next, o);
                next = fmaxf(fmaxf(next, n), fminf(best, b));
                best = fmaxf(best, b);
            }
            if (lane == 0) group_value[g] = group_of(best, next, a.group_best);
        }
        __syncthreads();
        const float value = lane < a.groups ? group_value[lane] : -INFINITY;
        const unsigned long long stay = groups_that_stay<64>(value, lane, 0, a.groups, a.top_groups);
        for (int e = t; e < a.experts; e += kRouteThreads)
            if (!(stay >> (e / per) & 1)) pick[e] = -INFINITY;
    }
    // the best of this thread's experts; found anew only by the thread that won
    float best = -INFINITY;
    int which = a.experts;
    const auto look = [&] {
        best = -INFINITY;
        which = a.experts;
        for (int e = t; e < a.experts; e += kRouteThreads)
            if (pick[e] > best) best = pick[e], which = e;
    };
    look();
    int at = -1;
    for (int j = 0; j < a.k; ++j) {
        float top = best;
        int won = which;
        for (int o = 1; o < 64; o <<= 1) {
            const float b = __shfl_xor(top, o);
            const int w = __shfl_xor(won, o);
            if (b > top || (b == top && w < won)) top = b, won = w;
        }
        if (lane == 0) part[wave] = top, where[wave] = won;
        __syncthreads();
        top = part[0], won = where[0];
#pragma unroll
        for (int w = 1; w < 4; ++w)
            if (part[w] > top || (part[w] == top && where[w] < won)) top = part[w], won = where[w];
        if (lane == j) at = top > -INFINITY ? won : -1;
        if (top > -INFINITY && which == won) {
            pick[won] = -INFINITY;
            look();
        }
        __syncthreads();
    }
    if (wave == 0) write_choices<T, 64>(a, row, lane, at, bad, low, total);
}

// Gradient of the scores.  LANES lanes a row: lane j works out choice j's part and
// puts it into the row in LDS, from where the row goes out once, V neighbours a
// lane; a softmax over the whole row is worked out again from the scores.  Bound by
// the write of the rows, and that read (65,536 bf16 rows of 256 experts: 12 us, 2.9 TB/s;
// with a wave to a row 19).  Rows of more than LANES V experts are taken in pieces of
// that many.
template <typename T, typename G, int LANES, int V>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(RouteArgs a) {
    constexpr int kRows = kRouteThreads / LANES, kWide = LANES * V;
    __shared__ __align__(16) float parts[kRows][kWide];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t row = (int64_t)blockIdx.x * kRows + slot;
    const bool there = row < a.n;
    const int64_t r = there ? row : a.n - 1;
    const T *s = static_cast<const T *>(a.scores) + r * a.lds;
    T *out = static_cast<T *>(a.dscores) + r * a.experts;
    float *mine = parts[slot];
    const int at = lane < a.k ? a.index[r * a.k + lane] : -1;
    const bool here = at >= 0 && at < a.experts;
    const float weight = lane < a.k ? a.weight[r * a.k + lane] : 0.f;
    float g = here ? (float)static_cast<const G *>(a.dweight)[r * a.k + lane] : 0.f;
    const bool bad = row_ballot<LANES>(weight != weight) != 0;
    const float score = here ? (float)s[at] : -INFINITY;
    float part;               // of the chosen score
    float mean = 0.f, low = 0.f, by_total = 1.f;
    const bool whole = a.softmax && !a.renormalise;
    float x[V];
    // the share of each choice in its row's sum (renormalised): exactly 1 where there
    // is one, so that its gradient is exactly 0
    const float share = a.scale != 0.f ? weight / a.scale : 0.f;
    const float inner = across_sum<LANES>(g * share);
    if (a.softmax) {
        mean = a.scale * inner;
        part = weight * (g - inner);
        if (whole) {
            low = -INFINITY;
            for (int e0 = lane * V; e0 < a.experts; e0 += kWide) {
                read_row<T, V>(s, e0, a.experts, -INFINITY, x);
#pragma unroll
                for (int v = 0; v < V; ++v) low = fmaxf(low, x[v]);
            }
            low = across_max<LANES>(low);
            low = low > -INFINITY ? low : 0.f;
            float total = 0.f;
            for (int e0 = lane * V; e0 < a.experts; e0 += kWide) {
                if (a.experts > kWide) read_row<T, V>(s, e0, a.experts, -INFINITY, x);
#pragma unroll
                for (int v = 0; v < V; ++v) total += expf(x[v] - low);
            }
            total = across_sum<LANES>(total);
            by_total = total > 0.f ? 1.f / total : 1.f;
            part = a.scale * g;
        }
    } else {
        const float p = here ? sigmoid(score) : 0.f;
        float by = a.scale;
        if (a.renormalise) {
            const float sum = across_sum<LANES>(p);
            by = sum > 0.f ? a.scale / sum : 0.f;
            g -= inner;
        }
        part = by * g * p * (1.f - p);
    }
    const float none = bad ? NAN : 0.f;
    for (int w0 = 0; w0 < a.experts; w0 += kWide) {
        const int e0 = w0 + lane * V;
#pragma unroll
        for (int v = 0; v < V; ++v) mine[lane * V + v] = none;
        // a row's lanes are in one wave
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (here && !bad && at >= w0 && at < w0 + kWide) mine[at - w0] = part;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = mine[lane * V + v];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (whole && e0 < a.experts) {
            if (a.experts > kWide) read_row<T, V>(s, e0, a.experts, -INFINITY, x);
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] = expf(x[v] - low) * by_total * (d[v] - mean);
        }
        if (there) write_row<T, V>(out, e0, a.experts, d);
    }
}

// --------------------------------------------------------------- dispatch
// A stable counting sort of the slots by expert.  Workgroup b takes the slots of
// chunk b, its waves a part each, in order, their experts in registers.  count: the
// chunk's slots per expert.  place: the rank of a slot among its wave's 64 comes
// from the lanes that hold the same expert; the waves and chunks before it are
// added.  Whole numbers only: the order does not depend on timing.
//
// Few chunks: every workgroup of place adds up the counts of the chunks itself
// (from the caches), which saves a launch; that grows with their square, so many
// chunks are added up once (scan).  Both calls, with and without scan: 32 chunks
// of 256 experts 12.1 and 10.5 us, 128 chunks 14.3 and 15.8, 2048 chunks 86 and 679;
// 32 chunks of 2048 experts 26 and 33.
constexpr int kFewChunks = 64, kFewCounts = 32768;
constexpr int kChunk = 4096, kSortThreads = 1024;

__device__ inline int expert_at(const DispatchArgs &a, int64_t s, int64_t end) {
    const int e = s < end ? a.index[s] : -1;
    return e >= 0 && e < a.experts ? e : -1;
}

__global__ __launch_bounds__(kSortThreads) void dispatch_count_kernel(DispatchArgs a) {
    extern __shared__ int hist[];
    for (int e = threadIdx.x; e < a.experts; e += kSortThreads) hist[e] = 0;
    __syncthreads();
    const int64_t s0 = (int64_t)blockIdx.x * kChunk;
    const int64_t end = s0 + kChunk < a.slots ? s0 + kChunk : a.slots;
    for (int64_t s = s0 + threadIdx.x; s < end; s += kSortThreads) {
        const int e = expert_at(a, s, end);
        if (e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kSortThreads)
        a.counts[(int64_t)blockIdx.x * a.experts + e] = hist[e];
}

// Replaces the counts by those of the chunks before, and writes the sums of all
// behind them.  A workgroup takes 64 experts, its waves a part of the chunks each.
__global__ __launch_bounds__(kSortThreads) void dispatch_scan_kernel(DispatchArgs a) {
    constexpr int kWaves = kSortThreads / 64;
    __shared__ int part[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e = blockIdx.x * 64 + lane;
    const int each = (a.blocks + kWaves - 1) / kWaves;
    const int b0 = wave * each, b1 = b0 + each < a.blocks ? b0 + each : a.blocks;
    int sum = 0;
    if (e < a.experts) {
#pragma unroll 8
        for (int b = b0; b < b1; ++b) sum += a.counts[(int64_t)b * a.experts + e];
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (e >= a.experts) return;
    int before = 0;
    for (int w = 0; w < wave; ++w) before += part[w][lane];
#pragma unroll 8
    for (int b = b0; b < b1; ++b) {
        int *at = a.counts + (int64_t)b * a.experts + e;
        const int c = *at;
        *at = before;
        before += c;
    }
    if (wave == kWaves - 1) a.counts[(int64_t)a.blocks * a.experts + e] = before;
}

// WAVES: waves that rank (fewer where their histograms do not fit in LDS: 524,288
// slots of 256 experts 14 us with 16, 18 with 4).
template <int WAVES>
__global__ __launch_bounds__(kSortThreads) void dispatch_place_kernel(DispatchArgs a) {
    constexpr int kPart = kChunk / WAVES, kHeld = kPart / 64;
    constexpr int kExperts = 256, kLanes = kSortThreads / kExperts;   // per pass over the experts
    extern __shared__ int base[];   // WAVES x experts
    __shared__ int sums[kExperts / 64], found[2][kLanes][kExperts];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t s0 = (int64_t)blockIdx.x * kChunk, w0 = s0 + (int64_t)wave * kPart;
    const int64_t end = s0 + kChunk < a.slots ? s0 + kChunk : a.slots;
    int *mine = base + wave * a.experts;
    int held[kHeld];
    if (wave < WAVES) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) held[h] = expert_at(a, w0 + h * 64 + lane, end);
    }
    for (int e = t; e < WAVES * a.experts; e += kSortThreads) base[e] = 0;
    __syncthreads();
    if (wave < WAVES && (WAVES > 1 || a.blocks == 1)) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
            if (held[h] >= 0) atomicAdd(&mine[held[h]], 1);
    }
    __syncthreads();
    // expert by expert, 256 at a time: the chunk's first row, then the waves'
    int before = 0;   // rows of the experts below these 256
    const int le = t % kExperts, part = t / kExperts;
    for (int e0 = 0; e0 < a.experts; e0 += kExperts) {
        const int e = e0 + le;
        int all = 0, prior = 0;
        if (e < a.experts) {
            if (a.blocks == 1) {
                for (int w = part; w < WAVES; w += kLanes) all += base[w * a.experts + e];
            } else if (a.scanned) {
                if (part == 0) {
                    all = a.counts[(int64_t)a.blocks * a.experts + e];
                    prior = a.counts[(int64_t)blockIdx.x * a.experts + e];
                }
            } else {
#pragma unroll 8
                for (int b = part; b < a.blocks; b += kLanes) {
                    const int c = a.counts[(int64_t)b * a.experts + e];
                    all += c;
                    prior += b < (int)blockIdx.x ? c : 0;
                }
            }
        }
        found[0][part][le] = all;
        found[1][part][le] = prior;
        __syncthreads();
        int sum = 0, first = 0;
        if (part == 0) {
            all = prior = 0;
#pragma unroll
            for (int l = 0; l < kLanes; ++l) all += found[0][l][le], prior += found[1][l][le];
            sum = all;   // inclusive over the lanes
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(sum, o);
                if (lane >= o) sum += v;
            }
            if (lane == 63) sums[wave] = sum;
        }
        __syncthreads();
        int next = before;
#pragma unroll
        for (int w = 0; w < kExperts / 64; ++w) next += sums[w];
        if (part == 0 && e < a.experts) {
            first = before + sum - all;
            for (int w = 0; w < wave; ++w) first += sums[w];
            if (blockIdx.x == 0) a.offsets[e] = first;
            int at = first + prior;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int c = base[w * a.experts + e];
                base[w * a.experts + e] = at;
                at += c;
            }
        }
        before = next;
        __syncthreads();
    }
    if (blockIdx.x == 0 && t == 0) a.offsets[a.experts] = before;
    for (int64_t p = before + (int64_t)blockIdx.x * kSortThreads + t; p < a.slots;
         p += (int64_t)gridDim.x * kSortThreads)
        a.order[p] = -1;
    if (wave >= WAVES) return;
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const int64_t s = w0 + h * 64 + lane;
        const int e = held[h];
        if (w0 + h * 64 >= end) break;
        // the lanes that hold the same expert
        unsigned long long same = __ballot(e >= 0);
        for (int b = 1; b < a.experts; b <<= 1) {
            const unsigned long long ones = __ballot(e & b);
            same &= e & b ? ones : ~ones;
        }
        if (e >= 0) {
            const int p = mine[e] + __popcll(same & ((1ull << lane) - 1));
            a.order[p] = (int)s;
            a.place[s] = p;
        } else if (s < end) {
            a.place[s] = -1;
        }
        // the wave's reads of the rows counted so far come before the leaders' writes
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (e >= 0 && __ffsll((long long)same) - 1 == lane) mine[e] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Up to kSortSlots slots, in one workgroup.
__global__ __launch_bounds__(kRouteThreads) void dispatch_few_kernel(DispatchArgs a) {
    __shared__ int expert[kSortSlots];
    if ((int)threadIdx.x < a.slots) expert[threadIdx.x] = expert_at(a, threadIdx.x, a.slots);
    __syncthreads();
    sort_few(a, expert);
}

// Lets a kernel have `bytes` of dynamic LDS where, with its own, they pass 64 KB.
template <typename K>
hipError_t room_for(K kernel, size_t bytes) {
    if (bytes <= 48 * 1024) return hipSuccess;
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T>
hipError_t launch_route_type(const RouteArgs &a, const DispatchArgs &sort, hipStream_t stream) {
    const bool wide = a.k > 16 || a.groups > 16;
    const auto blocks = [&](int rows) { return (unsigned)((a.n + rows - 1) / rows); };
    const auto lds = [&](int rows) {
        return a.groups > 1 ? (size_t)rows * (a.experts + 1) * sizeof(float) : 0;
    };
    if (a.experts <= 64 && !wide)
        route_kernel<T, 16, 4><<<blocks(16), kRouteThreads, lds(16), stream>>>(a, sort);
    else if (a.experts <= 256 && !wide)
        route_kernel<T, 16, 16><<<blocks(16), kRouteThreads, lds(16), stream>>>(a, sort);
    else if (a.experts <= 512)
        route_kernel<T, 64, 8><<<blocks(4), kRouteThreads, lds(4), stream>>>(a, sort);
    else if (a.experts <= 1024)
        route_kernel<T, 64, 16><<<blocks(4), kRouteThreads, lds(4), stream>>>(a, sort);
    else if (a.experts <= 2048)
        route_kernel<T, 64, 32><<<blocks(4), kRouteThreads, lds(4), stream>>>(a, sort);
    else {
        const hipError_t e = room_for(route_long_kernel<T>, a.experts * sizeof(float));
        if (e != hipSuccess) return e;
        route_long_kernel<T><<<(unsigned)a.n, kRouteThreads, a.experts * sizeof(float), stream>>>(a);
    }
    return hipGetLastError();
}

template <typename T, typename G>
hipError_t launch_backward_types(const RouteArgs &a, hipStream_t stream) {
    const auto blocks = [&](int rows) { return (unsigned)((a.n + rows - 1) / rows); };
    if (a.experts <= 64 && a.k <= 16)
        route_backward_kernel<T, G, 16, 4><<<blocks(16), kRouteThreads, 0, stream>>>(a);
    else if (a.experts <= 256 && a.k <= 16)
        route_backward_kernel<T, G, 16, 16><<<blocks(16), kRouteThreads, 0, stream>>>(a);
    else
        route_backward_kernel<T, G, 64, 8><<<blocks(4), kRouteThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_backward_type(const RouteArgs &a, hipStream_t stream) {
    switch (a.dweight_type) {
        case kF32: return launch_backward_types<T, float>(a, stream);
        case kBF16: return launch_backward_types<T, __bf16>(a, stream);
        default: return launch_backward_types<T, _Float16>(a, stream);
    }
}

}  // namespace

bool route_sorts(const RouteArgs &a) {
    const int rows = a.experts <= 256 && a.k <= 16 && a.groups <= 16 ? 16 : 4;  // of a workgroup
    return a.n > 0 && a.n <= rows && a.n * a.k <= kSortSlots && a.experts <= 2048;
}

// Launches `launch` on the call's rows, as many at a time as a grid of up to 256
// threads a row holds.
template <typename F>
static hipError_t in_rows(const RouteArgs &args, F launch) {
    constexpr int64_t kMost = (int64_t)1 << 23;
    const int64_t size = type_size(args.type), gsize = type_size(args.dweight_type);
    for (int64_t r = 0; r < args.n; r += kMost) {
        RouteArgs a = args;
        a.n = args.n - r < kMost ? args.n - r : kMost;
        a.scores = static_cast<const char *>(a.scores) + r * a.lds * size;
        a.index += r * a.k;
        a.weight += r * a.k;
        if (a.dweight) a.dweight = static_cast<const char *>(a.dweight) + r * a.k * gsize;
        if (a.dscores) a.dscores = static_cast<char *>(a.dscores) + r * a.experts * size;
        const hipError_t e = launch(a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_route(const RouteArgs &args, const DispatchArgs *sort, hipStream_t stream) {
    const DispatchArgs with = sort ? *sort : DispatchArgs{};
    return in_rows(args, [&](const RouteArgs &a) {
        switch (a.type) {
            case kF32: return launch_route_type<float>(a, with, stream);
            case kBF16: return launch_route_type<__bf16>(a, with, stream);
            default: return launch_route_type<_Float16>(a, with, stream);
        }
    });
}

hipError_t launch_route_backward(const RouteArgs &args, hipStream_t stream) {
    return in_rows(args, [&](const RouteArgs &a) {
        switch (a.type) {
            case kF32: return launch_backward_type<float>(a, stream);
            case kBF16: return launch_backward_type<__bf16>(a, stream);
            default: return launch_backward_type<_Float16>(a, stream);
        }
    });
}

int32_t dispatch_blocks(int64_t slots) {
    return slots <= kChunk ? 1 : (int32_t)((slots + kChunk - 1) / kChunk);
}

hipError_t launch_dispatch(const DispatchArgs &args, hipStream_t stream) {
    DispatchArgs a = args;
    const size_t one = a.experts * sizeof(int);
    if (a.slots <= kSortSlots) {
        dispatch_few_kernel<<<1, kRouteThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    a.scanned = a.blocks > kFewChunks || (int64_t)a.blocks * a.experts > kFewCounts;
    if (a.blocks > 1) {
        const hipError_t e = room_for(dispatch_count_kernel, one);
        if (e != hipSuccess) return e;
        dispatch_count_kernel<<<a.blocks, kSortThreads, one, stream>>>(a);
        if (a.scanned)
            dispatch_scan_kernel<<<(a.experts + 63) / 64, kSortThreads, 0, stream>>>(a);
    }
    if (a.experts <= 512)
        dispatch_place_kernel<16><<<a.blocks, kSortThreads, 16 * one, stream>>>(a);
    else if (a.experts <= 2048)
        dispatch_place_kernel<4><<<a.blocks, kSortThreads, 4 * one, stream>>>(a);
    else {
        const hipError_t e = room_for(dispatch_place_kernel<1>, one);
        if (e != hipSuccess) return e;
        dispatch_place_kernel<1><<<a.blocks, kSortThreads, one, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace som
