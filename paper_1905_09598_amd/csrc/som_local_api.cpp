// Host side of the local models: the C ABI declared in include/som_local.h.
// Validates every argument before any device work, lays out the caller's work
// memory, chooses how each product runs, and enqueues the kernels.
#include "som_local.h"
#include "som_internal.h"
#include "som_local_internal.h"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

namespace som {

// How a product runs.  Few rows: the kernel that streams w.  Otherwise the tile
// and the number of parts of the contraction with the least estimated time:
// rounds of workgroups over the compute units, slabs in each, and the pass that
// joins the parts.  aligned: whether both sides lie in whole 16-byte pieces.
ProductPlan plan_product(const ProductArgs &a, bool aligned, int num_cus) {
    ProductPlan best{};
    best.aligned = aligned;
    const int64_t experts = a.offsets ? a.experts : 1;
    const int64_t slab = a.eight ? 128 : 128 / type_size(a.type);
    const bool along = a.mode == kForward || a.mode == kPair;
    // a gated layer's tiles hold the same columns of two matrices
    const int64_t columns = a.mode == kPair ? 2 * a.n : a.n;
    if (along && a.m <= 16 * experts) {
        best.tile = 16;
        const int64_t groups = (a.n + 15) / 16 * std::min(a.m, a.m / best.tile + experts);
        // as few waves to a workgroup as keep the chip's loads in flight (16 waves of
        // four slabs a compute unit), so that all workgroups run at once
        best.waves = 4;
        const int64_t turn = a.eight ? 4 * slab : slab;   // of a wave
        while (best.waves < 16 && groups * best.waves < (int64_t)num_cus * 16 &&
               a.k > best.waves * turn)
            best.waves *= 2;
        best.splits = 1;
        return best;
    }
    // Microseconds of a slab on one workgroup that has a compute unit to itself and
    // on as many as it holds, by type; what unaligned rows add; a tile's start and
    // end.  Fitted to 39 products of 100 to 5000 rows, 100 to 9096 columns and
    // contractions of 100 to 8000, each timed in all shapes and splits, and checked on
    // 37 others of 120 to 16,001 rows: the chosen shape took 1.006 of the best one's
    // time on average, at most 1.10.
    struct Cost { double one, all, unaligned; };
    struct Shape { int32_t tile, held; Cost half, single; double ends; };
    static const Shape shapes[] = {{256, 1, {1.5, 1.5, 0.0}, {7.0, 7.0, 0.0}, 6.0},
                                   {128, 2, {0.8, 0.9, 0.25}, {2.0, 3.4, 0.1}, 4.5},
                                   {64, 4, {0.43, 0.78, 0.25}, {0.7, 1.7, 0.2}, 2.5}};
    static const int32_t splits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    best.time = INFINITY;
    for (const Shape &s : shapes) {
        if (!aligned && s.tile == 256) continue;
        const Cost &cost = a.type == kF32 ? s.single : s.half;
        const int64_t tn = (columns + s.tile - 1) / s.tile;
        int64_t tm, k = a.k;
        if (a.mode == kWeight) {
            tm = (a.m + s.tile - 1) / s.tile * experts;
            k = (a.k + experts - 1) / experts;
        } else {
            // an expert's last tile is half empty
            tm = a.offsets ? a.m / s.tile + (std::min(experts, a.m) + 1) / 2
                           : (a.m + s.tile - 1) / s.tile;
        }
        const int64_t slabs = std::max<int64_t>(1, (k + slab - 1) / slab);
        const int64_t rows = a.mode == kWeight ? a.m * experts : a.m;
        const int32_t most = a.mode == kGate ? 1 : 32;   // its rows' dots need whole sums
        for (const int32_t parts : splits) {
            if (parts > most || parts > slabs) break;
            const int64_t floats = parts > 1 ? parts * rows * (tn * s.tile) : 0;
            if (floats > (int64_t)1 << 30) break;
            const double groups = (double)(tm * tn * parts) / num_cus;   // to a compute unit
            // finding a tile's expert and its rows takes several reads in turn; a last
            // slab of unaligned rows is read element by element
            const double ends = s.ends + (a.offsets ? 8.0 : 0.0) + (aligned ? 0.0 : 1.0);
            // `held` workgroups at a time, one tile each
            const auto round = [&](double held) {
                const double more = s.held > 1 ? (cost.all - cost.one) * (held - 1) / (s.held - 1) : 0;
                return ((slabs + parts - 1) / parts) *
                           (cost.one + more + (aligned ? 0.0 : cost.unaligned)) + ends;
            };
            double time;
            if (groups > 4.0 * s.held) {
                time = (groups / s.held + 0.5) * round(s.held);
            } else {
                const int32_t whole = std::max(1, (int32_t)std::ceil(groups));
                time = whole / s.held * round(s.held);
                if (whole % s.held) time += round(whole % s.held);
            }
            if (parts > 1) time += 2.0 + 0.2 * parts + floats * 4.0 * (1 / 3.0e6 + 1 / 4.0e6);
            if (time < best.time) {
                best.time = time;
                best.tile = s.tile;
                best.splits = parts;
                best.partial_floats = floats;
            }
        }
    }
    return best;
}

}  // namespace som

namespace {

using som::ProductArgs;
using som::ProductPlan;

som_status from_hip(hipError_t e) {
    if (e == hipSuccess) return SOM_OK;
    if (e == hipErrorOutOfMemory || e == hipErrorMemoryAllocation) return SOM_E_OOM;
    if (e == hipErrorInvalidValue) return SOM_E_UNSUPPORTED;  // a grid beyond its limits
    return SOM_E_DEVICE;
}

bool type_ok(int32_t t) { return t == SOM_F32 || t == SOM_BF16 || t == SOM_F16; }
bool activation_ok(int32_t a) { return a >= SOM_ACT_NONE && a <= SOM_ACT_SILU; }

// rows rows of cols elements, ld apart, at p.
bool rows_ok(const void *p, int64_t rows, int64_t cols, int64_t ld, int size) {
    if (rows == 0 || cols == 0) return true;
    if (!p || ld < cols || reinterpret_cast<uintptr_t>(p) % size != 0) return false;
    unsigned __int128 elems = (unsigned __int128)(rows - 1) * (uint64_t)ld + (uint64_t)cols;
    if (elems > (unsigned __int128)1 << 56) return false;
    return som::device_range_ok(p, (uint64_t)elems * size);
}
bool rows_ok_or_null(const void *p, int64_t rows, int64_t cols, int64_t ld, int size) {
    return !p || rows_ok(p, rows, cols, ld, size);
}

int compute_units() {
    static int cus = [] {
        int dev = 0, v = 0;
        if (hipGetDevice(&dev) != hipSuccess ||
            hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) {
            (void)hipGetLastError();
            v = 256;
        }
        return v > 0 ? v : 256;
    }();
    return cus;
}

// Takes pieces of the caller's work memory, or, without one, adds up what they need.
struct Carver {
    char *base;
    uint64_t used = 0;
    explicit Carver(void *p) : base(static_cast<char *>(p)) {}
    template <typename T = void>
    T *take(uint64_t bytes) {
        char *at = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return reinterpret_cast<T *>(at);
    }
};

int64_t rounded(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// One side of a product as the caller has it, and how it is read.
struct SideRows {
    const void *p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    const int32_t **list = nullptr;  // names `listed` of the rows, list[r] / per
    som::Divider per;
    int64_t listed = 0;
    som::RowsArgs copy{};
    bool copied = false;

    // Whole 16-byte pieces.
    bool whole(int size) const {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % (16 / size) == 0 &&
               cols % (16 / size) == 0;
    }
    // Beyond the offsets of the tiles' kernels: these rows have to be copied, in
    // the order of the list if it is the listed matrix that is too long.
    bool far(int size) const { return list && *list && rows * ld * size >= (int64_t)1 << 32; }
    bool beyond(int size) const { return far(size) || !som::tile_reaches(ld, size); }
    double copy_time(int size) const { return 3.0 + (double)rows * cols * size * 2 / 4.0e6; }

    // A copy in whole pieces; with z, times act'(z).
    void make_copy(Carver &work, int32_t type, const void *z = nullptr, int32_t activation = 0) {
        const int size = som::type_size(type);
        const int64_t ldd = rounded(cols, 16 / size);
        const bool by_list = list && *list && rows * ldd * size >= (int64_t)1 << 32;
        const int64_t high = by_list ? listed : rows;
        copied = true;
        copy.type = type;
        copy.activation = activation;
        copy.src = p;
        copy.z = z;
        copy.dst = work.take((uint64_t)high * ldd * size);
        copy.rows = high;
        copy.cols = cols;
        copy.lds = ld;
        copy.ldz = cols;
        copy.ldd = ldd;
        copy.list = by_list ? *list : nullptr;
        copy.per = per;
        if (by_list) *list = nullptr;
        p = copy.dst, ld = ldd, rows = high;
    }
};

hipError_t launch_product(const ProductArgs &a, const ProductPlan &plan, hipStream_t s) {
    switch (a.type) {
        case SOM_F32: return som::launch_product_f32(a, plan, s);
        case SOM_BF16: return som::launch_product_bf16(a, plan, s);
        default: return som::launch_product_f16(a, plan, s);
    }
}

// One product of a call, planned, with its parts' memory.  Sides that are not
// whole are read as they are by the kernels that can, or copied first where that
// and the faster kernels take less time.
struct Product {
    ProductArgs a{};
    ProductPlan plan{};
    void place(Carver &work, SideRows &A, SideRows &B) {
        const int size = som::type_size(a.type);
        const auto needs = [&](const SideRows &s) { return !s.whole(size) && !s.copied; };
        plan = som::plan_product(a, !needs(A) && !needs(B), compute_units());
        if (!plan.waves) {
            if (A.beyond(size)) A.make_copy(work, a.type);
            if (B.beyond(size)) B.make_copy(work, a.type);
            double copies = 0.0;
            if (needs(A)) copies += A.copy_time(size);
            if (needs(B)) copies += B.copy_time(size);
            const ProductPlan whole = som::plan_product(a, true, compute_units());
            if (whole.time + copies < plan.time || copies == 0.0) {
                if (needs(A)) A.make_copy(work, a.type);
                if (needs(B)) B.make_copy(work, a.type);
                plan = whole;
            }
        }
        a.a = A.p, a.lda = A.ld;
        a.b = B.p, a.ldb = B.ld;
        a.batch_b = B.ld * (a.mode == som::kForward ? a.n : a.k);
        if (plan.splits > 1) {
            a.partial = work.take<float>((uint64_t)plan.partial_floats * 4);
            a.partial_rows = a.mode == som::kWeight ? a.m * (a.offsets ? a.experts : 1) : a.m;
        }
    }
};

// How it runs, as som_linear_route says it; 0 if it is not wanted.
int32_t tile_of(const Product &p, bool wanted = true) {
    return !wanted ? 0 : p.plan.waves || p.plan.aligned ? p.plan.tile : -p.plan.tile;
}

hipError_t run_copy(const SideRows &side, hipStream_t s) {
    return side.copied ? som::launch_rows_copy(side.copy, s) : hipSuccess;
}

hipError_t run(const Product &p, hipStream_t s) { return launch_product(p.a, p.plan, s); }

// Runs the steps of a call in order, up to the first that fails.
template <typename... Step>
hipError_t in_order(Step... steps) {
    hipError_t e = hipSuccess;
    (void)((e = steps(), e == hipSuccess) && ...);
    return e;
}

SideRows side(const void *p, int64_t rows, int64_t cols, int64_t ld) {
    SideRows s;
    s.p = p, s.rows = rows, s.cols = cols, s.ld = ld;
    return s;
}
// Rows named by the order of the slots: a product's *list is set, and cleared again
// where a copy in that order takes the rows' place.
void by_slot(SideRows &s, const int32_t **list, const int32_t *order, int32_t k, int64_t slots) {
    *list = order;
    s.list = list, s.per = som::Divider(k), s.listed = slots;
}

// What a call enqueues, over the caller's work memory.
struct LinearForward {
    SideRows x, w;
    Product product;
    LinearForward(const som_linear_call &c, Carver &work) {
        ProductArgs &a = product.a;
        a.mode = som::kForward;
        a.type = c.type;
        a.activation = c.activation;
        a.m = c.n, a.n = c.outer, a.k = c.inner;
        a.bias = c.bias;
        a.residual = c.residual, a.ldr = c.ldr;
        a.y = c.y, a.z = c.z;
        x = side(c.x, c.n, c.inner, c.ldx);
        w = side(c.w, c.outer, c.inner, c.inner);
        product.place(work, x, w);
    }
    void route(int32_t *tiles) const { tiles[0] = tile_of(product); }
    hipError_t enqueue(hipStream_t s) const {
        return in_order([&] { return run_copy(x, s); }, [&] { return run_copy(w, s); },
                        [&] { return run(product, s); });
    }
};

struct LinearBackward {
    SideRows x, w, dz;
    Product input, weight;
    som::SumsArgs sums{};
    bool has_input, has_weight, has_rows;
    LinearBackward(const som_linear_call &c, Carver &work) {
        has_input = c.dx != nullptr && c.n;
        has_weight = c.dw != nullptr;
        has_rows = c.n != 0;
        dz = side(c.dy, c.n, c.outer, c.lddy);
        if (c.activation != SOM_ACT_NONE) dz.make_copy(work, c.type, c.z, c.activation);
        if (has_input) {
            ProductArgs &a = input.a;
            a.mode = som::kInput;
            a.type = c.type;
            a.m = c.n, a.n = c.inner, a.k = c.outer;
                a.y = c.dx;
            w = side(c.w, c.outer, c.inner, c.inner);
            input.place(work, dz, w);
        }
        if (has_weight) {
            ProductArgs &a = weight.a;
            a.mode = som::kWeight;
            a.type = c.type;
            a.m = c.outer, a.n = c.inner, a.k = c.n;
                a.y = c.dw;
            x = side(c.x, c.n, c.inner, c.ldx);
            weight.place(work, dz, x);
        }
        if (c.dbias) {
            sums.type = c.type;
            sums.src = dz.p;
            sums.rows = c.n, sums.cols = c.outer, sums.ld = dz.ld;
            sums.out = c.dbias;
            sums.partial = work.take<float>((uint64_t)som::sums_partial(sums) * 4);
        }
    }
    void route(int32_t *tiles) const {
        tiles[0] = tile_of(input, has_input), tiles[1] = tile_of(weight, has_weight);
    }
    hipError_t enqueue(hipStream_t s) const {
        const auto copy = [&](const SideRows &r) { return has_rows ? run_copy(r, s) : hipSuccess; };
        return in_order([&] { return copy(dz); }, [&] { return copy(w); }, [&] { return copy(x); },
                        [&] { return has_input ? run(input, s) : hipSuccess; },
                        [&] { return has_weight ? run(weight, s) : hipSuccess; },
                        [&] { return sums.out ? som::launch_sums(sums, s) : hipSuccess; });
    }
};

// Rows of `width` values in 8 bits: of their codes and of their scales.
int64_t codes_of(int64_t width) { return rounded(width, 128); }
int64_t scales_of(int64_t width) { return rounded(width, 512) / 128; }

// x is brought to 8 bits first, unless it is there or has few and short rows.
struct Linear8 {
    ProductArgs a{};
    ProductPlan plan{};
    som::BlocksArgs blocks{};
    som::Rows8Args few{};
    bool first;
    Linear8(const som_linear8_call &c, Carver &work) {
        a.mode = som::kForward;
        a.eight = 1;
        a.type = c.type;
        a.activation = c.activation;
        a.m = c.n, a.n = c.outer, a.k = codes_of(c.inner);
        a.lda = a.ldb = a.k;
        a.ld_scale = scales_of(c.inner);
        a.a = c.x_codes, a.scale_a = static_cast<const unsigned char *>(c.x_scale);
        a.b = c.w_codes, a.scale_b = static_cast<const unsigned char *>(c.w_scale);
        a.bias = c.bias;
        a.residual = c.residual, a.ldr = c.ldr;
        a.y = c.y;
        plan = som::plan_product(a, true, compute_units());
        first = !c.x_codes && (!plan.waves || som::rows8_lds(a) > som::kRows8Lds);
        if (!c.x_codes && !first) few.x = c.x, few.ldx = c.ldx, few.width = c.inner;
        if (first) {
            blocks.type = c.type;
            blocks.n = c.n, blocks.width = c.inner;
            blocks.x = c.x, blocks.ldx = c.ldx;
            blocks.ld_codes = a.k, blocks.ld_scale = a.ld_scale;
            blocks.codes = work.take<unsigned char>((uint64_t)c.n * a.k);
            blocks.scale = work.take<unsigned char>((uint64_t)c.n * a.ld_scale);
            a.a = blocks.codes, a.scale_a = blocks.scale;
        }
        if (plan.splits > 1) {
            a.partial = work.take<float>((uint64_t)plan.partial_floats * 4);
            a.partial_rows = a.m;
        }
    }
    hipError_t enqueue(hipStream_t s) const {
        return in_order([&] { return first ? som::launch_to_blocks(blocks, s) : hipSuccess; },
                        [&] { return som::launch_product8(a, few, plan, s); });
    }
};

struct GatedForward {
    SideRows x, w;
    Product product;
    GatedForward(const som_gated_call &c, Carver &work) {
        ProductArgs &a = product.a;
        a.mode = som::kPair;
        a.type = c.type;
        a.activation = c.activation;
        a.m = c.n, a.n = c.hidden, a.k = c.inner;
        a.bias = c.bias;
        a.y = c.y, a.z = c.z;
        x = side(c.x, c.n, c.inner, c.ldx);
        w = side(c.w, 2 * (int64_t)c.hidden, c.inner, c.inner);
        product.place(work, x, w);
    }
    void route(int32_t *tiles) const { tiles[0] = tile_of(product); }
    hipError_t enqueue(hipStream_t s) const {
        return in_order([&] { return run_copy(x, s); }, [&] { return run_copy(w, s); },
                        [&] { return run(product, s); });
    }
};

// dz of both matrices side by side, n x 2 hidden, then the products of one layer of
// 2 hidden rows.
struct GatedBackward {
    SideRows x, w, dz;
    Product input, weight;
    som::GatedArgs slopes{};
    void *dbias;
    bool has_input, has_weight, has_rows;
    GatedBackward(const som_gated_call &c, Carver &work) {
        const int size = som::type_size(c.type);
        const int64_t both = 2 * (int64_t)c.hidden;
        has_rows = c.n != 0;
        has_input = c.dx != nullptr && c.n;
        has_weight = c.dw != nullptr;
        dbias = c.dbias;
        slopes.type = c.type, slopes.activation = c.activation;
        slopes.n = c.n, slopes.hidden = c.hidden;
        slopes.dy = c.dy, slopes.lddy = c.lddy;
        slopes.z = c.z;
        slopes.ldd = rounded(both, 16 / size);
        dz = side(work.take((uint64_t)c.n * slopes.ldd * size), c.n, both, slopes.ldd);
        dz.copied = true;   // in whole pieces
        slopes.dz = const_cast<void *>(dz.p);
        slopes.parts = som::gated_parts(slopes, compute_units());
        if (c.dbias) slopes.partial = work.take<float>((uint64_t)slopes.parts * both * 4);
        const int64_t largest = som::gated_largest(slopes);
        if (largest) {
            slopes.largest = work.take<float>((uint64_t)largest * 4);
            slopes.power = work.take<int32_t>(4);
            input.a.power = weight.a.power = slopes.power;
        }
        if (has_input) {
            ProductArgs &a = input.a;
            a.mode = som::kInput;
            a.type = c.type;
            a.m = c.n, a.n = c.inner, a.k = both;
            a.y = c.dx;
            w = side(c.w, both, c.inner, c.inner);
            input.place(work, dz, w);
        }
        if (has_weight) {
            ProductArgs &a = weight.a;
            a.mode = som::kWeight;
            a.type = c.type;
            a.m = both, a.n = c.inner, a.k = c.n;
            a.y = c.dw;
            x = side(c.x, c.n, c.inner, c.ldx);
            weight.place(work, dz, x);
        }
    }
    void route(int32_t *tiles) const {
        tiles[0] = tile_of(input, has_input), tiles[1] = tile_of(weight, has_weight);
    }
    hipError_t enqueue(hipStream_t s) const {
        const auto copy = [&](const SideRows &r) { return has_rows ? run_copy(r, s) : hipSuccess; };
        return in_order([&] { return som::launch_gated_slopes(slopes, s); },
                        [&] { return copy(w); }, [&] { return copy(x); },
                        [&] { return has_input ? run(input, s) : hipSuccess; },
                        [&] { return has_weight ? run(weight, s) : hipSuccess; },
                        [&] {
                            return dbias ? som::launch_join_parts(
                                               slopes.type, slopes.partial, slopes.parts, slopes.hidden,
                                               dbias,
                                               static_cast<char *>(dbias) +
                                                   slopes.hidden * som::type_size(slopes.type),
                                               s)
                                         : hipSuccess;
                        });
    }
};

// The experts' answers: the routed products, in fp32, then the join.
struct ExpertsForward {
    SideRows x, h, w1, w2;
    Product first, second;
    som::CombineArgs join{};
    bool two;
    ExpertsForward(const som_experts_call &c, Carver &work) {
        const int size = som::type_size(c.type);
        const int64_t slots = c.n * c.k;
        const som::Divider per(c.k);
        two = c.w2 != nullptr;
        float *const answers = work.take<float>((uint64_t)slots * c.outer * 4);
        void *const hidden = two ? work.take((uint64_t)slots * c.hidden * size) : nullptr;
        ProductArgs &a = first.a;
        a.mode = som::kForward;
        a.type = c.type;
        a.m = slots, a.n = c.hidden, a.k = c.inner;
        a.offsets = c.offsets, a.experts = c.experts, a.per = per;
        a.slots = c.order, a.gates = c.weight;
        a.bias = c.b1;
        a.activation = c.activation;
        a.wide = !two;
        a.y = two ? hidden : answers;
        a.z = c.z, a.scaled = c.scaled;
        x = side(c.x, c.n, c.inner, c.ldx);
        by_slot(x, &a.list, c.order, c.k, slots);
        w1 = side(c.w1, (int64_t)c.experts * c.hidden, c.inner, c.inner);
        first.place(work, x, w1);
        if (two) {
            ProductArgs &b = second.a;
            b.mode = som::kForward;
            b.type = c.type;
            b.m = slots, b.n = c.outer, b.k = c.hidden;
            b.offsets = c.offsets, b.experts = c.experts, b.per = per;
            b.bias = c.b2;
            b.wide = 1;
            b.y = answers;
            h = side(hidden, slots, c.hidden, c.hidden);
            w2 = side(c.w2, (int64_t)c.experts * c.outer, c.hidden, c.hidden);
            second.place(work, h, w2);
        }
        join.type = c.type, join.k = c.k;
        join.n = c.n, join.width = c.outer;
        join.y = answers, join.weight = c.weight, join.place = c.place;
        join.residual = c.residual, join.ldr = c.ldr;
        join.out = c.y;
    }
    void route(int32_t *tiles) const { tiles[0] = tile_of(first), tiles[1] = tile_of(second, two); }
    hipError_t enqueue(hipStream_t s) const {
        return in_order([&] { return run_copy(x, s); }, [&] { return run_copy(w1, s); },
                        [&] { return run(first, s); },
                        [&] { return two ? run_copy(h, s) : hipSuccess; },
                        [&] { return two ? run_copy(w2, s) : hipSuccess; },
                        [&] { return two ? run(second, s) : hipSuccess; },
                        [&] { return som::launch_combine(join, s); });
    }
};

// Their gradients.  The last layer (w2, or w1 alone) takes its gradient from the
// documents' rows of dy, found by slot, and the weights come in after the sums:
//     C = w^T dy,  dweight = <C, u> + <dy, bias>  with u the layer's input,
//     the input's gradient g C (times the slope), dw = dy (g u)^T,
// with g u as forward kept it; in fp16 the power of two of a small weight is with dy, and
// local linear maps, which keep nothing, take all of g with dy: both in a copy of dy's
// rows by slot (4000 rows of 2000 in fp16: 8 us, of 640 for the whole training pass).
struct ExpertsBackward {
    SideRows dy_gate, dy_weight, w_last, scaled, dz_rows, w1, x;
    Product gate, last_weight, input, first_weight;
    som::SumsArgs last_sums{}, first_sums{};
    som::CombineArgs join{};
    som::DweightArgs dweight{};
    bool two, has_rows, has_gate, has_sums, has_input;
    ExpertsBackward(const som_experts_call &c, Carver &work) {
        const int size = som::type_size(c.type);
        const int64_t slots = c.n * c.k;
        const som::Divider per(c.k);
        two = c.w2 != nullptr;
        has_rows = slots != 0;
        const int32_t width = two ? c.hidden : c.inner;   // of the last layer's input
        const bool first = two && (c.dw1 || c.db1 || c.dx);
        has_gate = has_rows && (c.dweight || first || (!two && c.dx));
        has_input = has_rows && two && c.dx;
        void *dz = nullptr;
        float *parts = nullptr;
        if (c.dx) parts = work.take<float>((uint64_t)slots * c.inner * 4);
        if (has_gate) {
            ProductArgs &a = gate.a;
            a.mode = som::kGate;
            a.type = c.type;
            a.m = slots, a.n = width, a.k = c.outer;
            a.offsets = c.offsets, a.experts = c.experts, a.per = per;
            a.slots = c.order, a.gates = c.weight;
            a.activation = two ? c.activation : SOM_ACT_NONE;
            a.argument = two ? c.z : c.x;
            a.ld_argument = two ? c.hidden : c.ldx;
            a.argument_listed = !two;
            a.image = two && c.dweight && size == 2 ? c.scaled : nullptr;
            a.wide = !two;
            if (two) dz = work.take((uint64_t)slots * c.hidden * size);
            // without dx of local linear maps the products' rows are not wanted
            if (!two && !c.dx) parts = work.take<float>((uint64_t)slots * c.inner * 4);
            a.y = two ? dz : parts;
            dy_gate = side(c.dy, c.n, c.outer, c.lddy);
            by_slot(dy_gate, &a.list, c.order, c.k, slots);
            w_last = side(two ? c.w2 : c.w1, (int64_t)c.experts * c.outer, width, width);
            gate.place(work, dy_gate, w_last);
            a.dot_cols = som::plan_dot_cols(gate.plan, a.n);
            a.dots = work.take<float>((uint64_t)slots * a.dot_cols * 4);
        }
        void *const dw_last = two ? c.dw2 : c.dw1, *const db_last = two ? c.db2 : c.db1;
        const void *const b_last = two ? c.b2 : c.b1;
        if (dw_last) {
            ProductArgs &a = last_weight.a;
            a.mode = som::kWeight;
            a.type = c.type;
            a.m = c.outer, a.n = width, a.k = slots;
            a.offsets = c.offsets, a.experts = c.experts, a.per = per;
            a.y = dw_last;
            dy_weight = side(c.dy, c.n, c.outer, c.lddy);
            scaled = side(two ? c.scaled : c.x, two ? slots : c.n, width, two ? width : c.ldx);
            if (!two || (c.type == SOM_F16 && c.weight)) {
                dy_weight.rows = slots;
                dy_weight.make_copy(work, c.type);
                dy_weight.copy.list = c.order;
                dy_weight.copy.per = per;
                dy_weight.copy.gates = c.weight;
                dy_weight.copy.exponents = two;
                if (!two) by_slot(scaled, &a.list, c.order, c.k, slots);
            } else {
                a.list_of_a = 1;
                by_slot(dy_weight, &a.list, c.order, c.k, slots);
            }
            last_weight.place(work, dy_weight, scaled);
        }
        has_sums = db_last || (c.dweight && b_last);
        if (has_sums) {
            som::SumsArgs &s = last_sums;
            s.type = c.type;
            s.src = c.dy;
            s.rows = slots, s.cols = c.outer, s.ld = c.lddy;
            s.offsets = c.offsets, s.experts = c.experts;
            s.list = c.order, s.per = per, s.gates = c.weight;
            s.out = db_last;
            s.partial = work.take<float>((uint64_t)som::sums_partial(s) * 4);
            if (c.dweight && b_last) {
                s.bias = b_last;
                s.dot_cols = som::sums_dot_cols(s);
                s.dots = work.take<float>((uint64_t)slots * s.dot_cols * 4);
            }
        }
        dweight.type = c.type;
        dweight.slots = slots;
        dweight.place = c.place;
        dweight.dots[0] = gate.a.dots, dweight.cols[0] = gate.a.dot_cols;
        dweight.dots[1] = last_sums.dots, dweight.cols[1] = last_sums.dot_cols;
        dweight.dweight = c.dweight;
        dz_rows = side(dz, slots, c.hidden, c.hidden);
        if (two && c.dw1) {
            ProductArgs &a = first_weight.a;
            a.mode = som::kWeight;
            a.type = c.type;
            a.m = c.hidden, a.n = c.inner, a.k = slots;
            a.offsets = c.offsets, a.experts = c.experts, a.per = per;
            a.y = c.dw1;
            x = side(c.x, c.n, c.inner, c.ldx);
            by_slot(x, &a.list, c.order, c.k, slots);
            first_weight.place(work, dz_rows, x);
        }
        if (two && c.db1) {
            som::SumsArgs &s = first_sums;
            s.type = c.type;
            s.src = dz;
            s.rows = slots, s.cols = c.hidden, s.ld = c.hidden;
            s.offsets = c.offsets, s.experts = c.experts;
            s.out = c.db1;
            s.partial = work.take<float>((uint64_t)som::sums_partial(s) * 4);
        }
        if (has_input) {
            ProductArgs &a = input.a;
            a.mode = som::kInput;
            a.type = c.type;
            a.m = slots, a.n = c.inner, a.k = c.hidden;
            a.offsets = c.offsets, a.experts = c.experts, a.per = per;
            a.wide = 1;
            a.y = parts;
            w1 = side(c.w1, (int64_t)c.experts * c.hidden, c.inner, c.inner);
            input.place(work, dz_rows, w1);
        }
        join.type = c.type, join.k = c.k;
        join.n = c.n, join.width = c.inner;
        join.y = parts, join.place = c.place;
        join.out = c.dx;
    }
    void route(int32_t *tiles) const {
        tiles[0] = tile_of(gate, has_gate), tiles[1] = tile_of(last_weight, last_weight.a.y);
        tiles[2] = tile_of(input, has_input), tiles[3] = tile_of(first_weight, first_weight.a.y);
    }
    hipError_t enqueue(hipStream_t s) const {
        const auto copy = [&](const SideRows &r) { return has_rows ? run_copy(r, s) : hipSuccess; };
        const auto product = [&](bool wanted, const Product &p) {
            return wanted ? run(p, s) : hipSuccess;
        };
        return in_order(
            [&] { return copy(dy_gate); }, [&] { return copy(w_last); },
            [&] { return product(has_gate, gate); },
            [&] { return copy(dy_weight); }, [&] { return copy(scaled); },
            [&] { return product(last_weight.a.y, last_weight); },
            [&] { return has_sums ? som::launch_sums(last_sums, s) : hipSuccess; },
            [&] { return dweight.dweight ? som::launch_dweight(dweight, s) : hipSuccess; },
            [&] { return copy(dz_rows); }, [&] { return copy(x); },
            [&] { return product(first_weight.a.y, first_weight); },
            [&] { return first_sums.out ? som::launch_sums(first_sums, s) : hipSuccess; },
            [&] { return copy(w1); },
            [&] { return product(has_input, input); },
            [&] { return join.out ? som::launch_combine(join, s) : hipSuccess; });
    }
};

// The sizes and types of a call; the pointers are checked apart, where a call
// is about to run.
som_status linear_sizes_ok(const som_linear_call *c) {
    if (!c || !type_ok(c->type) || !activation_ok(c->activation) || c->n < 0 || c->inner <= 0 ||
        c->outer <= 0 || c->ldx < c->inner)
        return SOM_E_ARG;
    if (c->inner > som::kMaxWidth || c->outer > som::kMaxWidth || c->n > (int64_t)1 << 40)
        return SOM_E_UNSUPPORTED;
    return SOM_OK;
}

som_status experts_sizes_ok(const som_experts_call *c) {
    if (!c || !type_ok(c->type) || !activation_ok(c->activation) || c->n < 0 || c->k < 1 ||
        c->experts < 1 || c->inner < 1 || c->hidden < 1 || c->outer < 1 || c->ldx < c->inner)
        return SOM_E_ARG;
    if (!c->w2 && (c->b2 || c->z || c->scaled || c->dw2 || c->db2 || c->outer != c->hidden ||
                   c->activation != SOM_ACT_NONE))
        return SOM_E_ARG;
    if (c->inner > som::kMaxWidth || c->hidden > som::kMaxWidth || c->outer > som::kMaxWidth ||
        (__int128)c->n * c->k > INT32_MAX || c->experts > som::kMaxExperts ||
        (int64_t)c->experts * std::max(c->hidden, c->outer) > INT32_MAX)
        return SOM_E_UNSUPPORTED;
    return SOM_OK;
}

// The call as it will run: the routing's arrays, which it needs, may not be there yet
// when its work memory is asked for.
som_experts_call routed(const som_experts_call &c) {
    static const int32_t there = 0;
    som_experts_call r = c;
    if (!r.offsets) r.offsets = &there;
    if (!r.order) r.order = &there;
    if (!r.place) r.place = &there;
    return r;
}

bool experts_common_ok(const som_experts_call &c) {
    const int size = som::type_size(c.type);
    const int64_t slots = c.n * c.k, e = c.experts;
    return rows_ok(c.x, c.n, c.inner, c.ldx, size) &&
           rows_ok(c.w1, e * c.hidden, c.inner, c.inner, size) &&
           rows_ok_or_null(c.b1, e, c.hidden, c.hidden, size) &&
           rows_ok_or_null(c.w2, e * c.outer, c.hidden, c.hidden, size) &&
           rows_ok_or_null(c.b2, e, c.outer, c.outer, size) &&
           rows_ok_or_null(c.weight, 1, slots, slots, 4) &&
           rows_ok(c.offsets, 1, e + 1, e + 1, 4) && rows_ok(c.order, 1, slots, slots, 4) &&
           rows_ok(c.place, 1, slots, slots, 4);
}

som_status work_ok(const Carver &need, void *workspace, uint64_t bytes) {
    if (need.used == 0) return SOM_OK;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || bytes < need.used ||
        !som::device_range_ok(workspace, need.used))
        return SOM_E_ARG;
    return SOM_OK;
}

// Lays a call out over its work memory, once to see what it needs, and enqueues it.
template <typename Plan, typename Call>
som_status enqueue(const Call &c) {
    Carver need(nullptr);
    Plan(c, need);
    const som_status st = work_ok(need, c.workspace, c.workspace_bytes);
    if (st != SOM_OK) return st;
    Carver work(c.workspace);
    return from_hip(Plan(c, work).enqueue(reinterpret_cast<hipStream_t>(c.stream)));
}

template <typename Forward, typename Backward, typename Call>
uint64_t workspace(const Call &c, bool backward) {
    Carver need(nullptr);
    if (backward) Backward(c, need);
    else Forward(c, need);
    return need.used;
}

template <typename Forward, typename Backward, typename Call>
void route(const Call &c, bool backward, int32_t *tiles, int32_t count) {
    std::fill(tiles, tiles + count, 0);
    Carver need(nullptr);
    if (c.n == 0) return;
    if (backward) Backward(c, need).route(tiles);
    else Forward(c, need).route(tiles);
}

}  // namespace

extern "C" {

som_status som_linear_workspace(const som_linear_call *c, int32_t backward, uint64_t *bytes) {
    if (!bytes) return SOM_E_ARG;
    const som_status st = linear_sizes_ok(c);
    if (st == SOM_OK) *bytes = c->n ? workspace<LinearForward, LinearBackward>(*c, backward) : 0;
    return st;
}

som_status som_linear_route(const som_linear_call *c, int32_t backward, int32_t tiles[2]) {
    if (!tiles) return SOM_E_ARG;
    const som_status st = linear_sizes_ok(c);
    if (st == SOM_OK) route<LinearForward, LinearBackward>(*c, backward, tiles, 2);
    return st;
}

som_status som_linear(const som_linear_call *c) {
    const som_status st = linear_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    if (!rows_ok(c->w, c->outer, c->inner, c->inner, size) ||
        !rows_ok(c->x, c->n, c->inner, c->ldx, size) ||
        !rows_ok(c->y, c->n, c->outer, c->outer, size) ||
        !rows_ok_or_null(c->z, c->n, c->outer, c->outer, size) ||
        !rows_ok_or_null(c->bias, 1, c->outer, c->outer, size) ||
        !rows_ok_or_null(c->residual, c->n, c->outer, c->ldr, size))
        return SOM_E_ARG;
    return c->n ? enqueue<LinearForward>(*c) : SOM_OK;
}

som_status som_linear_backward(const som_linear_call *c) {
    const som_status st = linear_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    if (!rows_ok(c->w, c->outer, c->inner, c->inner, size) ||
        !rows_ok(c->x, c->n, c->inner, c->ldx, size) ||
        !rows_ok(c->dy, c->n, c->outer, c->lddy, size) ||
        (c->activation != SOM_ACT_NONE && !rows_ok(c->z, c->n, c->outer, c->outer, size)) ||
        !rows_ok_or_null(c->dx, c->n, c->inner, c->inner, size) ||
        !rows_ok_or_null(c->dw, c->outer, c->inner, c->inner, size) ||
        !rows_ok_or_null(c->dbias, 1, c->outer, c->outer, size))
        return SOM_E_ARG;
    return enqueue<LinearBackward>(*c);
}

static som_status gated_sizes_ok(const som_gated_call *c) {
    if (!c || !type_ok(c->type) || !activation_ok(c->activation) || c->n < 0 || c->inner <= 0 ||
        c->hidden <= 0 || c->ldx < c->inner)
        return SOM_E_ARG;
    if (c->inner > som::kMaxWidth || c->hidden > som::kMaxWidth / 2 || c->n > (int64_t)1 << 40)
        return SOM_E_UNSUPPORTED;
    return SOM_OK;
}

static bool gated_common_ok(const som_gated_call &c) {
    const int size = som::type_size(c.type);
    return rows_ok(c.w, 2 * (int64_t)c.hidden, c.inner, c.inner, size) &&
           rows_ok(c.x, c.n, c.inner, c.ldx, size);
}

som_status som_gated_workspace(const som_gated_call *c, int32_t backward, uint64_t *bytes) {
    if (!bytes) return SOM_E_ARG;
    const som_status st = gated_sizes_ok(c);
    if (st == SOM_OK)
        *bytes = c->n || backward ? workspace<GatedForward, GatedBackward>(*c, backward) : 0;
    return st;
}

som_status som_gated_route(const som_gated_call *c, int32_t backward, int32_t tiles[2]) {
    if (!tiles) return SOM_E_ARG;
    const som_status st = gated_sizes_ok(c);
    if (st == SOM_OK) route<GatedForward, GatedBackward>(*c, backward, tiles, 2);
    return st;
}

som_status som_gated(const som_gated_call *c) {
    const som_status st = gated_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int64_t both = 2 * (int64_t)c->hidden;
    const int size = som::type_size(c->type);
    if (!gated_common_ok(*c) || !rows_ok(c->y, c->n, c->hidden, c->hidden, size) ||
        !rows_ok_or_null(c->z, c->n, both, both, 4) || !rows_ok_or_null(c->bias, 1, both, both, size))
        return SOM_E_ARG;
    return c->n ? enqueue<GatedForward>(*c) : SOM_OK;
}

som_status som_gated_backward(const som_gated_call *c) {
    const som_status st = gated_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int64_t both = 2 * (int64_t)c->hidden;
    const int size = som::type_size(c->type);
    if (!gated_common_ok(*c) || !rows_ok(c->dy, c->n, c->hidden, c->lddy, size) ||
        !rows_ok(c->z, c->n, both, both, 4) ||
        !rows_ok_or_null(c->dx, c->n, c->inner, c->inner, size) ||
        !rows_ok_or_null(c->dw, both, c->inner, c->inner, size) ||
        !rows_ok_or_null(c->dbias, 1, both, both, size))
        return SOM_E_ARG;
    return enqueue<GatedBackward>(*c);
}

som_status som_experts_workspace(const som_experts_call *c, int32_t backward, uint64_t *bytes) {
    if (!bytes) return SOM_E_ARG;
    const som_status st = experts_sizes_ok(c);
    if (st == SOM_OK) *bytes = c->n ? workspace<ExpertsForward, ExpertsBackward>(routed(*c), backward) : 0;
    return st;
}

som_status som_experts_route(const som_experts_call *c, int32_t backward, int32_t tiles[4]) {
    if (!tiles) return SOM_E_ARG;
    const som_status st = experts_sizes_ok(c);
    if (st == SOM_OK) route<ExpertsForward, ExpertsBackward>(routed(*c), backward, tiles, 4);
    return st;
}

som_status som_experts(const som_experts_call *c) {
    const som_status st = experts_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    const int64_t slots = c->n * c->k;
    if ((c->z != nullptr) != (c->scaled != nullptr)) return SOM_E_ARG;
    if (!experts_common_ok(*c) || !rows_ok(c->y, c->n, c->outer, c->outer, size) ||
        !rows_ok_or_null(c->z, slots, c->hidden, c->hidden, size) ||
        !rows_ok_or_null(c->scaled, slots, c->hidden, c->hidden, size) ||
        !rows_ok_or_null(c->residual, c->n, c->outer, c->ldr, size))
        return SOM_E_ARG;
    return c->n ? enqueue<ExpertsForward>(*c) : SOM_OK;
}

som_status som_experts_backward(const som_experts_call *c) {
    const som_status st = experts_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    const int64_t slots = c->n * c->k, e = c->experts;
    if (!experts_common_ok(*c) || !rows_ok(c->dy, c->n, c->outer, c->lddy, size) ||
        (c->w2 && (!rows_ok(c->z, slots, c->hidden, c->hidden, size) ||
                   !rows_ok(c->scaled, slots, c->hidden, c->hidden, size))) ||
        !rows_ok_or_null(c->dx, c->n, c->inner, c->inner, size) ||
        !rows_ok_or_null(c->dweight, c->n, c->k, c->k, size) ||
        !rows_ok_or_null(c->dw1, e * c->hidden, c->inner, c->inner, size) ||
        !rows_ok_or_null(c->db1, e, c->hidden, c->hidden, size) ||
        !rows_ok_or_null(c->dw2, e * c->outer, c->hidden, c->hidden, size) ||
        !rows_ok_or_null(c->db2, e, c->outer, c->outer, size))
        return SOM_E_ARG;
    return enqueue<ExpertsBackward>(*c);
}

// Codes and scales of rows rows of `width` values.
static bool blocks_ok(const void *codes, const void *scale, int64_t rows, int64_t width) {
    const int64_t c = codes_of(width), s = scales_of(width);
    return rows_ok(codes, rows, c, c, 1) && rows_ok(scale, rows, s, s, 1) &&
           (rows == 0 || (reinterpret_cast<uintptr_t>(codes) % 16 == 0 &&
                          reinterpret_cast<uintptr_t>(scale) % 4 == 0));
}

som_status som_to_blocks(const som_blocks_call *c) {
    if (!c || !type_ok(c->type) || c->n < 0 || c->width < 1 || c->ldx < c->width) return SOM_E_ARG;
    if (c->width > som::kMaxWidth || c->n > (int64_t)1 << 40) return SOM_E_UNSUPPORTED;
    if (!rows_ok(c->x, c->n, c->width, c->ldx, som::type_size(c->type)) ||
        !blocks_ok(c->codes, c->scale, c->n, c->width))
        return SOM_E_ARG;
    som::BlocksArgs a{};
    a.type = c->type;
    a.n = c->n, a.width = c->width;
    a.x = c->x, a.ldx = c->ldx;
    a.codes = static_cast<unsigned char *>(c->codes), a.ld_codes = codes_of(c->width);
    a.scale = static_cast<unsigned char *>(c->scale), a.ld_scale = scales_of(c->width);
    return from_hip(som::launch_to_blocks(a, reinterpret_cast<hipStream_t>(c->stream)));
}

static som_status linear8_sizes_ok(const som_linear8_call *c) {
    if (!c || (c->type != SOM_BF16 && c->type != SOM_F16) || !activation_ok(c->activation) ||
        c->n < 0 || c->inner <= 0 || c->outer <= 0 || (c->n && !c->x_codes && c->ldx < c->inner))
        return SOM_E_ARG;
    if (c->inner > som::kMaxWidth || c->outer > som::kMaxWidth || c->n > (int64_t)1 << 40)
        return SOM_E_UNSUPPORTED;
    return SOM_OK;
}

som_status som_linear8_workspace(const som_linear8_call *c, uint64_t *bytes) {
    if (!bytes) return SOM_E_ARG;
    const som_status st = linear8_sizes_ok(c);
    if (st == SOM_OK) {
        Carver need(nullptr);
        if (c->n) Linear8(*c, need);
        *bytes = need.used;
    }
    return st;
}

som_status som_linear8_route(const som_linear8_call *c, int32_t route[2]) {
    if (!route) return SOM_E_ARG;
    const som_status st = linear8_sizes_ok(c);
    if (st != SOM_OK) return st;
    route[0] = route[1] = 0;
    if (c->n) {
        Carver need(nullptr);
        const Linear8 call(*c, need);
        route[0] = call.plan.tile, route[1] = call.plan.splits;
    }
    return SOM_OK;
}

som_status som_linear8(const som_linear8_call *c) {
    const som_status st = linear8_sizes_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    if ((c->x_codes ? c->x != nullptr || !blocks_ok(c->x_codes, c->x_scale, c->n, c->inner)
                    : c->x_scale != nullptr || !rows_ok(c->x, c->n, c->inner, c->ldx, size)) ||
        !blocks_ok(c->w_codes, c->w_scale, c->outer, c->inner) ||
        !rows_ok(c->y, c->n, c->outer, c->outer, size) ||
        !rows_ok_or_null(c->bias, 1, c->outer, c->outer, size) ||
        !rows_ok_or_null(c->residual, c->n, c->outer, c->ldr, size))
        return SOM_E_ARG;
    return c->n ? enqueue<Linear8>(*c) : SOM_OK;
}

static som_status norm_ok(const som_norm_call *c) {
    if (!c || !type_ok(c->type) || c->n < 0 || c->width < 1 || c->ldx < c->width ||
        !(c->eps >= 0.f) || isinf(c->eps))
        return SOM_E_ARG;
    if (c->width > som::kMaxWidth || c->n > (int64_t)1 << 40) return SOM_E_UNSUPPORTED;
    return SOM_OK;
}

static som::NormArgs norm_args(const som_norm_call &c) {
    som::NormArgs a{};
    a.type = c.type;
    a.n = c.n, a.width = c.width;
    a.x = c.x, a.ldx = c.ldx;
    a.weight = c.weight, a.bias = c.bias;
    a.eps = c.eps;
    a.y = c.y, a.kept = c.kept;
    a.dy = c.dy, a.lddy = c.lddy;
    a.beside = c.beside, a.ldb = c.ldb;
    a.dx = c.dx, a.dweight = c.dweight, a.dbias = c.dbias;
    if (c.dweight || c.dbias) a.parts = som::norm_parts(a, compute_units());
    return a;
}

// The work memory of backward.
static void norm_place(som::NormArgs &a, Carver &work) {
    a.partial = work.take<float>((uint64_t)a.parts * 2 * a.width * 4);
    if (som::norm_long_columns(a)) a.off = work.take<float>((uint64_t)a.n * 4);
}

static bool norm_common_ok(const som_norm_call &c) {
    const int size = som::type_size(c.type);
    return rows_ok(c.x, c.n, c.width, c.ldx, size) &&
           rows_ok_or_null(c.weight, 1, c.width, c.width, size);
}

som_status som_norm_workspace(const som_norm_call *c, int32_t backward, uint64_t *bytes) {
    if (!bytes) return SOM_E_ARG;
    const som_status st = norm_ok(c);
    if (st == SOM_OK) {
        Carver need(nullptr);
        som::NormArgs a = norm_args(*c);
        if (backward) norm_place(a, need);
        *bytes = need.used;
    }
    return st;
}

som_status som_norm(const som_norm_call *c) {
    const som_status st = norm_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    if (!norm_common_ok(*c) || !rows_ok_or_null(c->bias, 1, c->width, c->width, size) ||
        !rows_ok(c->y, c->n, c->width, c->width, size) || !rows_ok_or_null(c->kept, c->n, 2, 2, 4))
        return SOM_E_ARG;
    if (c->n == 0) return SOM_OK;
    return from_hip(som::launch_norm(norm_args(*c), compute_units(),
                                     reinterpret_cast<hipStream_t>(c->stream)));
}

som_status som_norm_backward(const som_norm_call *c) {
    const som_status st = norm_ok(c);
    if (st != SOM_OK) return st;
    const int size = som::type_size(c->type);
    if (!norm_common_ok(*c) || !rows_ok(c->kept, c->n, 2, 2, 4) ||
        !rows_ok(c->dy, c->n, c->width, c->lddy, size) ||
        !rows_ok_or_null(c->beside, c->n, c->width, c->ldb, size) ||
        !rows_ok_or_null(c->dx, c->n, c->width, c->width, size) ||
        !rows_ok_or_null(c->dweight, 1, c->width, c->width, size) ||
        !rows_ok_or_null(c->dbias, 1, c->width, c->width, size))
        return SOM_E_ARG;
    Carver work(c->workspace);
    som::NormArgs a = norm_args(*c);
    norm_place(a, work);
    const som_status ok = work_ok(work, c->workspace, c->workspace_bytes);
    if (ok != SOM_OK) return ok;
    if (!a.parts && (c->n == 0 || !c->dx)) return SOM_OK;
    return from_hip(som::launch_norm_backward(a, compute_units(),
                                              reinterpret_cast<hipStream_t>(c->stream)));
}

som_status som_distill(const som_distill_call *c) {
    if (!c || !type_ok(c->type) || c->n < 0 || c->classes < 1 || c->lds < c->classes || c->k < 0 ||
        c->k > som::kMaxTaught ||
        !(c->temperature >= som::kLeastTemperature && c->temperature <= 1.f / som::kLeastTemperature) ||
        !(c->mix >= 0.f && c->mix <= 1.f) || !isfinite(c->scale))
        return SOM_E_ARG;
    if ((c->k && !type_ok(c->teacher_type)) || (!c->k && (c->index || c->teacher || c->rest)) ||
        (!c->k && c->mix != 0.f) || (c->n && !c->label && c->mix != 1.f))
        return SOM_E_ARG;
    if (c->classes > som::kMaxClasses || c->n > (int64_t)1 << 40) return SOM_E_UNSUPPORTED;
    const int size = som::type_size(c->type);
    if (!rows_ok(c->logits, c->n, c->classes, c->lds, size) ||
        !rows_ok_or_null(c->rest, 1, c->n, c->n, 4) || !rows_ok_or_null(c->label, 1, c->n, c->n, 4) ||
        !rows_ok_or_null(c->dloss, 1, c->n, c->n, 4) || !rows_ok_or_null(c->loss, 1, c->n, c->n, 4) ||
        !rows_ok_or_null(c->dlogits, c->n, c->classes, c->classes, size))
        return SOM_E_ARG;
    if (c->k && (!rows_ok(c->index, c->n, c->k, c->k, 4) ||
                 !rows_ok(c->teacher, c->n, c->k, c->k, som::type_size(c->teacher_type))))
        return SOM_E_ARG;
    if (c->n == 0 || (!c->loss && !c->dlogits)) return SOM_OK;
    // in the logits' place a row is read before it is written, beside them another's are not
    if (c->dlogits && (c->dlogits != c->logits || (c->lds != c->classes && c->n > 1))) {
        const char *const from = static_cast<const char *>(c->logits);
        const char *const to = static_cast<const char *>(c->dlogits);
        if (to < from + ((c->n - 1) * c->lds + c->classes) * size && from < to + c->n * c->classes * size)
            return SOM_E_ARG;
    }
    som::DistillArgs a{};
    a.type = c->type, a.teacher_type = c->teacher_type;
    a.n = c->n, a.classes = c->classes;
    a.k = c->mix == 0.f ? 0 : c->k;
    a.logits = c->logits, a.lds = c->lds;
    a.index = c->index, a.teacher = c->teacher, a.rest = c->rest;
    a.label = c->label;
    a.temperature = c->temperature, a.mix = c->mix;
    a.dloss = c->dloss, a.scale = c->scale;
    a.loss = c->loss, a.dlogits = c->dlogits;
    return from_hip(som::launch_distill(a, reinterpret_cast<hipStream_t>(c->stream)));
}

static som_status route_ok(const som_route_call *c) {
    if (!c || !type_ok(c->type) || (c->gate != SOM_GATE_SOFTMAX && c->gate != SOM_GATE_SIGMOID))
        return SOM_E_ARG;
    if (c->n < 0 || c->experts < 1 || c->experts > som::kMaxExperts || c->k < 1 ||
        c->k > std::min(c->experts, som::kMaxChoices))
        return SOM_E_ARG;
    if (c->groups < 1 || c->groups > som::kMaxGroups || c->experts % c->groups != 0 ||
        c->top_groups < 1 || c->top_groups > c->groups || c->group_best < 1 || c->group_best > 2)
        return SOM_E_ARG;
    if (!isfinite(c->scale) || c->lds < c->experts) return SOM_E_ARG;
    if ((__int128)c->n * c->k > INT32_MAX) return SOM_E_UNSUPPORTED;
    if (!rows_ok(c->scores, c->n, c->experts, c->lds, som::type_size(c->type)) ||
        !rows_ok(c->index, c->n, c->k, c->k, 4) || !rows_ok(c->weight, c->n, c->k, c->k, 4) ||
        !rows_ok_or_null(c->bias, 1, c->experts, c->experts, 4))
        return SOM_E_ARG;
    return SOM_OK;
}

static som::RouteArgs route_args(const som_route_call &c) {
    som::RouteArgs a{};
    a.type = c.type;
    a.softmax = c.gate == SOM_GATE_SOFTMAX;
    a.n = c.n;
    a.experts = c.experts;
    a.k = c.k;
    a.groups = c.groups;
    a.top_groups = c.top_groups;
    a.group_best = c.group_best;
    a.renormalise = c.renormalise != 0;
    a.scale = c.scale;
    a.scores = c.scores;
    a.lds = c.lds;
    a.bias = c.bias;
    a.index = c.index;
    a.weight = c.weight;
    a.dweight = c.dweight;
    a.dweight_type = c.dweight_type;
    a.dscores = c.dscores;
    return a;
}

som_status som_route_backward(const som_route_call *c) {
    const som_status st = route_ok(c);
    if (st != SOM_OK) return st;
    if (!type_ok(c->dweight_type) ||
        !rows_ok(c->dweight, c->n, c->k, c->k, som::type_size(c->dweight_type)) ||
        !rows_ok(c->dscores, c->n, c->experts, c->experts, som::type_size(c->type)))
        return SOM_E_ARG;
    return from_hip(
        som::launch_route_backward(route_args(*c), reinterpret_cast<hipStream_t>(c->stream)));
}

som_status som_dispatch_workspace(int64_t n, int32_t k, int32_t experts, uint64_t *bytes) {
    if (!bytes || n < 0 || k < 1 || experts < 1 || experts > som::kMaxExperts) return SOM_E_ARG;
    if ((__int128)n * k > INT32_MAX) return SOM_E_UNSUPPORTED;
    const int32_t blocks = som::dispatch_blocks(n * k);
    *bytes = blocks > 1 ? ((uint64_t)blocks + 1) * experts * 4 : 0;
    return SOM_OK;
}

static bool dispatch_ok(int64_t n, int32_t k, int32_t experts, const int32_t *offsets,
                        const int32_t *order, const int32_t *place, const void *work,
                        uint64_t work_bytes, uint64_t need) {
    return rows_ok(offsets, 1, experts + 1, experts + 1, 4) && rows_ok(order, n, k, k, 4) &&
           rows_ok(place, n, k, k, 4) &&
           (!need || (work_bytes >= need && rows_ok(work, 1, need / 4, need / 4, 4)));
}

static som::DispatchArgs dispatch_args(const int32_t *index, int64_t n, int32_t k,
                                       int32_t experts, int32_t *offsets, int32_t *order,
                                       int32_t *place, void *work) {
    som::DispatchArgs a{};
    a.index = index;
    a.slots = n * k;
    a.experts = experts;
    a.offsets = offsets;
    a.order = order;
    a.place = place;
    a.counts = static_cast<int32_t *>(work);
    a.blocks = som::dispatch_blocks(a.slots);
    return a;
}

som_status som_dispatch(const int32_t *index, int64_t n, int32_t k, int32_t experts,
                        int32_t *offsets, int32_t *order, int32_t *place, void *work,
                        uint64_t work_bytes, void *stream) {
    uint64_t need = 0;
    const som_status st = som_dispatch_workspace(n, k, experts, &need);
    if (st != SOM_OK) return st;
    if (!rows_ok(index, n, k, k, 4) ||
        !dispatch_ok(n, k, experts, offsets, order, place, work, work_bytes, need))
        return SOM_E_ARG;
    return from_hip(som::launch_dispatch(
        dispatch_args(index, n, k, experts, offsets, order, place, work),
        reinterpret_cast<hipStream_t>(stream)));
}

som_status som_route(const som_route_call *c) {
    const som_status st = route_ok(c);
    if (st != SOM_OK) return st;
    uint64_t need = 0;
    if (c->offsets) {
        (void)som_dispatch_workspace(c->n, c->k, c->experts, &need);
        if (!dispatch_ok(c->n, c->k, c->experts, c->offsets, c->order, c->place, c->workspace,
                         c->workspace_bytes, need))
            return SOM_E_ARG;
    }
    const hipStream_t s = reinterpret_cast<hipStream_t>(c->stream);
    const som::DispatchArgs sort = dispatch_args(c->index, c->n, c->k, c->experts, c->offsets,
                                                 c->order, c->place, c->workspace);
    const som::RouteArgs a = route_args(*c);
    const bool together = c->offsets && som::route_sorts(a);
    return from_hip(in_order(
        [&] { return som::launch_route(a, together ? &sort : nullptr, s); },
        [&] { return c->offsets && !together ? som::launch_dispatch(sort, s) : hipSuccess; }));
}

}  // extern "C"

// ------------------------------------------------------------------ AdamW
struct som_adamw {
    int device = 0;
    int32_t bits = 32, count = 0;
    std::vector<int64_t> counts;         // elements of each tensor
    std::vector<int32_t> first_chunk;    // of each launch of up to kAdamwGrads tensors
    som::AdamwChunk *chunks = nullptr;   // device
    som::AdamwTensor *tensors = nullptr; // device
    void *mean = nullptr, *square = nullptr;
    float *mean_scale = nullptr, *square_scale = nullptr, *master = nullptr;
};

extern "C" {

int64_t som_adamw_room(const som_adamw_tensor *tensors, int32_t count) {
    if (!tensors || count < 0) return -1;
    int64_t room = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (tensors[i].count < 0 || tensors[i].count > (int64_t)1 << 48) return -1;
        room += rounded(tensors[i].count, som::kAdamwBlock);
    }
    return room;
}

som_status som_adamw_destroy(som_adamw *opt) {
    if (!opt) return SOM_OK;
    hipError_t e = hipSuccess;
    if (opt->chunks) e = hipFree(opt->chunks);
    if (opt->tensors) {
        const hipError_t f = hipFree(opt->tensors);
        if (e == hipSuccess) e = f;
    }
    delete opt;
    return from_hip(e);
}

static som_status adamw_create(const som_adamw_tensor *tensors, int32_t count, int32_t bits,
                               void *mean, void *square, float *mean_scale, float *square_scale,
                               float *master, som_adamw **out) {
    const int64_t room = som_adamw_room(tensors, count);
    const int64_t blocks = room / som::kAdamwBlock;
    const int size = bits == 8 ? 1 : 4;
    if (!rows_ok(mean, 1, room, room, size) || !rows_ok(square, 1, room, room, size) ||
        !rows_ok_or_null(master, 1, room, room, 4))
        return SOM_E_ARG;
    // read four elements at a time, from multiples of four
    const uintptr_t all = reinterpret_cast<uintptr_t>(mean) | reinterpret_cast<uintptr_t>(square);
    if (all % (4 * size) != 0 || reinterpret_cast<uintptr_t>(master) % 16 != 0) return SOM_E_ARG;
    if (bits == 8 && (!rows_ok(mean_scale, 1, blocks, blocks, 4) ||
                      !rows_ok(square_scale, 1, blocks, blocks, 4)))
        return SOM_E_ARG;
    std::vector<som::AdamwChunk> chunks;
    std::vector<som::AdamwTensor> table;
    som_adamw *o = new som_adamw;
    *out = o;   // released by the caller on failure
    o->bits = bits;
    o->count = count;
    o->mean = mean, o->square = square;
    o->mean_scale = mean_scale, o->square_scale = square_scale, o->master = master;
    constexpr int32_t kStep = som::kAdamwChunk / som::kAdamwBlock;
    int64_t state = 0;
    for (int32_t i = 0; i < count; ++i) {
        const som_adamw_tensor &t = tensors[i];
        if (!type_ok(t.type) ||
            (t.count && !rows_ok(t.param, 1, t.count, t.count, som::type_size(t.type))))
            return SOM_E_ARG;
        if (i % som::kAdamwGrads == 0) o->first_chunk.push_back((int32_t)chunks.size());
        const int64_t nblocks = rounded(t.count, som::kAdamwBlock) / som::kAdamwBlock;
        if (nblocks > INT32_MAX - kStep ||
            (int64_t)chunks.size() + nblocks / kStep + 1 > INT32_MAX)
            return SOM_E_UNSUPPORTED;
        for (int64_t b = 0; b < nblocks; b += kStep)
            chunks.push_back({i % som::kAdamwGrads, (int32_t)b});
        table.push_back({t.param, t.count, state, t.type, 0});
        o->counts.push_back(t.count);
        state += nblocks * som::kAdamwBlock;
    }
    o->first_chunk.push_back((int32_t)chunks.size());
    hipError_t e = hipGetDevice(&o->device);
    if (!chunks.empty()) {
        const size_t cb = chunks.size() * sizeof(chunks[0]), tb = table.size() * sizeof(table[0]);
        if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void **>(&o->chunks), cb);
        if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void **>(&o->tensors), tb);
        if (e == hipSuccess) e = hipMemcpy(o->chunks, chunks.data(), cb, hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipMemcpy(o->tensors, table.data(), tb, hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipDeviceSynchronize();
    }
    return from_hip(e);
}

som_status som_adamw_create(const som_adamw_tensor *tensors, int32_t count, int32_t bits,
                            void *mean, void *square, float *mean_scale, float *square_scale,
                            float *master, som_adamw **out) {
    if (!out) return SOM_E_ARG;
    *out = nullptr;
    if (som_adamw_room(tensors, count) < 0 || count == 0 || (bits != 8 && bits != 32))
        return SOM_E_ARG;
    if ((bits == 8) != (mean_scale != nullptr) || (bits == 8) != (square_scale != nullptr))
        return SOM_E_ARG;
    som_adamw *o = nullptr;
    som_status st;
    try {
        st = adamw_create(tensors, count, bits, mean, square, mean_scale, square_scale, master, &o);
    } catch (const std::bad_alloc &) {
        st = SOM_E_OOM;
    } catch (...) {
        st = SOM_E_DEVICE;
    }
    if (st != SOM_OK) {
        (void)som_adamw_destroy(o);
        return st;
    }
    *out = o;
    return SOM_OK;
}

som_status som_adamw_step(som_adamw *o, const void *const *grads, const int32_t *grad_types,
                          int64_t step, double lr, double beta1, double beta2, double eps,
                          double weight_decay, void *stream) {
    if (!o || !grads || !grad_types || step < 1) return SOM_E_ARG;
    if (!(lr >= 0.0) || !(eps >= 0.0) || !(weight_decay >= 0.0) || isinf(lr) || isinf(eps) ||
        isinf(weight_decay) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
        return SOM_E_ARG;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return SOM_E_DEVICE;
    if (dev != o->device) return SOM_E_ARG;
    for (int32_t i = 0; i < o->count; ++i) {
        if (!type_ok(grad_types[i])) return SOM_E_ARG;
        if (!rows_ok(grads[i], 1, o->counts[i], o->counts[i], som::type_size(grad_types[i])))
            return SOM_E_ARG;
    }
    som::AdamwArgs a{};
    a.mean = o->mean, a.square = o->square;
    a.mean_scale = o->mean_scale, a.square_scale = o->square_scale;
    a.master = o->master;
    a.beta1 = (float)beta1;
    a.rest1 = (float)(1.0 - beta1);
    a.beta2 = (float)beta2;
    a.rest2 = (float)(1.0 - beta2);
    a.decay = (float)(1.0 - lr * weight_decay);
    a.rate = (float)(lr / (1.0 - pow(beta1, (double)step)));
    a.root_scale = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    a.eps = (float)eps;
    for (int32_t l = 0; l * som::kAdamwGrads < o->count; ++l) {
        const int32_t t0 = l * som::kAdamwGrads;
        const int32_t tensors = std::min(o->count - t0, (int32_t)som::kAdamwGrads);
        for (int32_t i = 0; i < tensors; ++i) {
            a.grads[i] = grads[t0 + i];
            a.grad_type[i] = (unsigned char)grad_types[t0 + i];
        }
        a.chunks = o->chunks + o->first_chunk[l];
        a.tensors = o->tensors + t0;
        a.nchunks = o->first_chunk[l + 1] - o->first_chunk[l];
        const hipError_t e = som::launch_adamw(a, o->bits == 8,
                                               reinterpret_cast<hipStream_t>(stream));
        if (e != hipSuccess) return from_hip(e);
    }
    return SOM_OK;
}

}  // extern "C"
