// Host side of the Newton-Schulz entry points of include/lamb_ops.h: plans
// (validation, tile lists, workspace) and the launches of a call.
#include <math.h>

#include <algorithm>

#include "ops_host.h"
#include "ortho_internal.h"

using namespace lamb_mi355x;

struct TileList {
    NsTile *tiles = nullptr;
    int32_t n = 0;
};

struct lamb_ns_plan {
    int device = 0;
    bool muon = false, bf16_in = false, split = false;
    NsKind kind = kNsBf16Out;
    int sym_shape = 0, update_shape = 0;
    int32_t blocks = 0;
    void *block = nullptr;  // every device buffer of the plan
    NsMatrix *matrices = nullptr;
    int32_t *block_matrix = nullptr;
    // of all matrices ([0]) and of those without chains ([1])
    TileList sym[2], update[2];
    TileList both, only_q, only_t, next_gram;  // of those with: Q and T, Q, T, A
    double *partials = nullptr;
    uint32_t *flag = nullptr;  // see launch_ns_check
    CallOrder order;
};

namespace {

constexpr int64_t kMaxSide = int64_t(1) << 20;

// The bounds of lamb_ns_params: where singular values that start in [0, 1] go.
lamb_status check_params(const lamb_ns_params &p) {
    if (p.reserved != 0)
        return fail(LAMB_EINVAL, "ns.reserved must be 0");
    if (p.steps < 1 || p.steps > 64)
        return fail(LAMB_EINVAL, "ns.steps = %d, need 1 to 64", p.steps);
    if (!std::isfinite(p.a) || !std::isfinite(p.b) || !std::isfinite(p.c))
        return fail(LAMB_EINVAL, "ns coefficients must be finite");
    if (!(p.eps >= 0.0f) || !std::isfinite(p.eps))
        return fail(LAMB_EINVAL, "ns.eps = %g, need finite and >= 0", double(p.eps));
    const double a = p.a, b = p.b, c = p.c;
    double top = 1.0;
    for (int k = 0; k < p.steps; ++k) {
        // extremes over t = s^2 in [0, top^2] of p(t) = a + b t + c t^2 and of
        // s p(s^2): the ends and the roots of the derivatives
        const double end = top * top;
        double largest_p = 0.0, largest_x = 0.0;
        auto look = [&](double t) {
            if (!(t >= 0.0 && t <= end))
                return;
            const double v = a + t * (b + t * c);
            largest_p = std::max(largest_p, std::fabs(v));
            largest_x = std::max(largest_x, std::sqrt(t) * std::fabs(v));
        };
        look(0.0);
        look(end);
        if (c != 0.0) {
            look(-b / (2.0 * c));
            const double d = 9.0 * b * b - 20.0 * a * c;  // a + 3 b t + 5 c t^2 = 0
            if (d >= 0.0) {
                look((-3.0 * b + std::sqrt(d)) / (10.0 * c));
                look((-3.0 * b - std::sqrt(d)) / (10.0 * c));
            }
        } else if (b != 0.0) {
            look(-a / (3.0 * b));
        }
        // the last result is not an operand again, but is held to the same bound
        if (!(largest_p <= kNsLargest) || !(largest_x <= kNsLargestX))
            return fail(LAMB_EINVAL,
                        "ns coefficients %g, %g, %g let the polynomial reach %.3g (at most %g) or "
                        "a singular value %.3g (at most %g) in step %d",
                        a, b, c, largest_p, kNsLargest, largest_x, kNsLargestX, k + 1);
        top = largest_x;
    }
    return LAMB_OK;
}

// The tile shape of a product is the one whose estimated time is least: the longest
// tile alone, or all tiles' time over the CUs, whichever is more. Microseconds, from
// lists of 1 to 1024 tiles with k = 1024 and 4096 on one GPU: a tile's fixed part, and
// its time per 1024 of k on a CU by itself and where all CUs work.
struct TileCost {
    double fixed, alone, full;
};
constexpr TileCost kCost[2][3] = {{{2.0, 3.7, 4.2}, {4.0, 8.6, 9.0}, {15.0, 17.5, 23.0}},
                                  {{2.5, 8.5, 8.5}, {3.5, 19.8, 24.5}, {18.0, 58.0, 77.0}}};
constexpr double kCus = 256.0;

struct Estimate {
    TileCost cost;
    double longest = 0.0, total = 0.0;
    void add(double tiles, double depth) {
        longest = std::max(longest, cost.fixed + depth / 1024.0 * cost.alone);
        total += tiles * (cost.fixed + depth / 1024.0 * cost.full);
    }
    double time() const { return std::max(longest, total / kCus); }
};

void pick_shapes(const std::vector<NsMatrix> &matrices, bool split, int *sym, int *update) {
    double best_sym = 1e300, best_update = 1e300;
    for (int shape = kNsTiny; shape <= kNsLarge; ++shape) {
        const double t = ns_tile(shape);
        Estimate gram{kCost[split][shape]}, poly{kCost[split][shape]}, up{kCost[split][shape]};
        for (const NsMatrix &m : matrices) {
            const double side = std::min(m.rows, m.cols), length = std::max(m.rows, m.cols);
            const double across = std::ceil(side / t);
            gram.add(across * (across + 1) / 2, length);
            poly.add(across * (across + 1) / 2, side);
            up.add(across * std::ceil(length / t), side);
        }
        const double time_sym = gram.time() + poly.time();
        if (time_sym < best_sym)
            best_sym = time_sym, *sym = shape;
        if (up.time() < best_update)
            best_update = up.time(), *update = shape;
    }
}

template <class F>
void for_tiles(int32_t rows, int32_t cols, int shape, F f) {
    const int64_t t = ns_tile(shape);
    for (int32_t r = 0; r * t < rows; ++r)
        for (int32_t c = 0; c * t < cols; ++c) f(r, c);
}

// Chains pay for matrices at least twice as long as wide, where they save more than
// their launches cost: BERT-Large's matrices (split, a third of them
// 1024 x 4096 or turned) take 15.0 ms a Muon step with chains and 18.6 without,
// ResNet-50's 1.00 and 1.16. Where the estimate says no: four matrices up to 256 x 1024
// would take 111 us in place of 94 (16-bit), a list around one of 2048 x 2048 979 in place
// of 900 (split).
void pick_chains(std::vector<NsMatrix> &matrices, bool split) {
    constexpr double kFlopsPerUs = 1e9, kChainUs = 100.0;
    const double turns = split ? kNsChainSplit : kNsChainHalf;
    double saved = 0.0;
    for (NsMatrix &m : matrices) {
        const double s = std::min(m.rows, m.cols), l = std::max(m.rows, m.cols);
        m.chain = l >= 2.0 * s;
        // for five iterations: three products of X each, or per chain, and four or so of
        // the short side
        if (m.chain)
            saved += 5.0 * s * s * (3.0 * l + s) - (5.0 / turns) * 3.0 * l * s * s -
                     5.0 * 3.0 * s * s * s;
    }
    if (saved * (split ? 3.0 : 1.0) < kChainUs * kFlopsPerUs)
        for (NsMatrix &m : matrices) m.chain = 0;
}

// Fills in sizes, tiles and workspace; `matrices` has its user's fields set.
lamb_status build(lamb_ns_plan *plan, std::vector<NsMatrix> &matrices) {
    pick_shapes(matrices, plan->split, &plan->sym_shape, &plan->update_shape);
    pick_chains(matrices, plan->split);
    std::vector<int32_t> block_matrix;
    int64_t elems = 0, blocks = 0;  // workspace, in 16-bit elements
    std::vector<int64_t> at_x(matrices.size()), at_gram(matrices.size());
    const int parts = plan->split ? 2 : 1;
    for (size_t i = 0; i < matrices.size(); ++i) {
        NsMatrix &m = matrices[i];
        m.tall = m.rows > m.cols;
        m.side = std::min(m.rows, m.cols);
        m.ld = int32_t(round_up(m.cols, 8));
        m.side_ld = int32_t(round_up(m.side, 8));
        m.x_low = round_up(int64_t(m.rows) * m.ld, 64);
        m.gram_low = round_up(int64_t(m.side) * m.side_ld, 64);
        at_x[i] = elems;
        elems += 2 * parts * m.x_low;
        at_gram[i] = elems;
        elems += (m.chain ? 6 : 2) * parts * m.gram_low;
        const int64_t units = int64_t(m.rows) * (m.ld / 8);
        const int64_t count = (units + kNsBlockUnits - 1) / kNsBlockUnits;
        if (blocks + count > INT32_MAX)
            return fail(LAMB_EINVAL, "the matrices hold too many elements for one plan");
        m.first_block = int32_t(blocks);
        m.blocks = int32_t(count);
        blocks += count;
        block_matrix.insert(block_matrix.end(), size_t(count), int32_t(i));
    }
    plan->blocks = int32_t(blocks);

    // Longest products first, so that the last workgroups are short ones.
    std::vector<int32_t> by_length(matrices.size()), by_side;
    for (size_t i = 0; i < by_length.size(); ++i) by_length[i] = int32_t(i);
    by_side = by_length;
    auto longest = [&](int32_t i) { return std::max(matrices[i].rows, matrices[i].cols); };
    std::stable_sort(by_length.begin(), by_length.end(),
                     [&](int32_t p, int32_t q) { return longest(p) > longest(q); });
    std::stable_sort(by_side.begin(), by_side.end(), [&](int32_t p, int32_t q) {
        return matrices[p].side > matrices[q].side;
    });
    enum Which { kAll, kDirect, kChained };
    auto wanted = [&](int32_t i, Which which) {
        return which == kAll || (matrices[i].chain != 0) == (which == kChained);
    };
    auto triangles = [&](const std::vector<int32_t> &order, Which which, int products, int first) {
        std::vector<NsTile> list;
        for (int32_t i : order)
            if (wanted(i, which))
                for (int32_t p = first; p < first + products; ++p)
                    for_tiles(matrices[i].side, matrices[i].side, plan->sym_shape,
                              [&](int32_t r, int32_t c) {
                                  if (c <= r)
                                      list.push_back(NsTile{i, r, c, p});
                              });
        return list;
    };
    auto whole = [&](Which which) {
        std::vector<NsTile> list;
        for (int32_t i : by_side)
            if (wanted(i, which))
                for_tiles(matrices[i].rows, matrices[i].cols, plan->update_shape,
                          [&](int32_t r, int32_t c) { list.push_back(NsTile{i, r, c, 0}); });
        return list;
    };
    std::vector<NsTile> lists[] = {triangles(by_length, kAll, 1, 0),
                                   triangles(by_length, kDirect, 1, 0),
                                   whole(kAll),
                                   whole(kDirect),
                                   triangles(by_side, kChained, 2, kNsQ),
                                   triangles(by_side, kChained, 1, kNsQ),
                                   triangles(by_side, kChained, 1, kNsT),
                                   triangles(by_side, kChained, 1, kNsA)};
    TileList *const held[] = {&plan->sym[0], &plan->sym[1], &plan->update[0], &plan->update[1],
                              &plan->both,   &plan->only_q, &plan->only_t,    &plan->next_gram};
    constexpr int kLists = sizeof held / sizeof held[0];
    static_assert(sizeof lists / sizeof lists[0] == kLists, "a place for every list");

    size_t bytes = 0;
    auto take = [&](size_t size) {
        const size_t at = bytes;
        bytes += size_t(round_up(int64_t(size), 256));
        return at;
    };
    const size_t o_work = take(size_t(elems) * 2);
    const size_t o_matrices = take(matrices.size() * sizeof(NsMatrix));
    const size_t o_blocks = take(block_matrix.size() * 4);
    size_t o_lists[kLists];
    for (int k = 0; k < kLists; ++k) {
        if (lists[k].size() > INT32_MAX)
            return fail(LAMB_EINVAL, "the matrices take too many tiles for one plan");
        o_lists[k] = take(lists[k].size() * sizeof(NsTile));
    }
    const size_t o_partials = take(size_t(blocks) * 8);
    const size_t o_flag = take(8);
    hipError_t err = hipGetDevice(&plan->device);
    if (err != hipSuccess)
        return fail_hip(err, "hipGetDevice");
    // only orders kernels of this device: no system-scope fence
    err = hipEventCreateWithFlags(&plan->order.done,
                                  hipEventDisableTiming | hipEventDisableSystemFence);
    if (err != hipSuccess)
        return fail_hip(err, "hipEventCreateWithFlags");
    err = hipMalloc(&plan->block, bytes);
    if (err != hipSuccess) {
        plan->block = nullptr;
        (void)hipGetLastError();
        return fail(LAMB_ENOMEM, "hipMalloc of %zu bytes: %s", bytes, hipGetErrorString(err));
    }
    char *base = static_cast<char *>(plan->block);
    uint16_t *work = reinterpret_cast<uint16_t *>(base + o_work);
    for (size_t i = 0; i < matrices.size(); ++i) {
        NsMatrix &m = matrices[i];
        m.x[0] = work + at_x[i];
        m.x[1] = m.x[0] + parts * m.x_low;
        auto square = [&](int k) { return work + at_gram[i] + k * parts * m.gram_low; };
        m.gram[0] = square(0);
        m.poly[0] = square(1);
        if (m.chain) {
            m.gram[1] = square(2);
            m.poly[1] = square(3);
            m.q = square(4);
            m.t = square(5);
        }
    }
    plan->matrices = reinterpret_cast<NsMatrix *>(base + o_matrices);
    plan->block_matrix = reinterpret_cast<int32_t *>(base + o_blocks);
    plan->partials = reinterpret_cast<double *>(base + o_partials);
    plan->flag = reinterpret_cast<uint32_t *>(base + o_flag);
    auto up = [&](void *to, const void *from, size_t size) {
        if (err == hipSuccess && size)
            err = hipMemcpy(to, from, size, hipMemcpyHostToDevice);
    };
    up(plan->matrices, matrices.data(), matrices.size() * sizeof(NsMatrix));
    up(plan->block_matrix, block_matrix.data(), block_matrix.size() * 4);
    for (int k = 0; k < kLists; ++k) {
        const std::vector<NsTile> spread = spread_over_dies(lists[k]);
        held[k]->tiles = reinterpret_cast<NsTile *>(base + o_lists[k]);
        held[k]->n = int32_t(spread.size());
        up(held[k]->tiles, spread.data(), spread.size() * sizeof(NsTile));
    }
    const uint32_t zero[2] = {};
    up(plan->flag, zero, sizeof zero);
    if (err != hipSuccess)
        return fail_hip(err, "hipMemcpy");
    return LAMB_OK;
}

lamb_status run(lamb_ns_plan *plan, const lamb_ns_params &ns, NsStep step, uint32_t *flag,
                int32_t *nonfinite_out, hipStream_t stream) {
    step.a = ns.a;
    step.b = ns.b;
    step.c = ns.c;
    step.eps = ns.eps;
    hipError_t err = launch_ns_norms(plan->matrices, plan->block_matrix, plan->blocks, plan->muon,
                                     plan->bf16_in, step, plan->partials, flag, nonfinite_out,
                                     stream);
    if (err == hipSuccess)
        err = launch_ns_convert(plan->matrices, plan->block_matrix, plan->blocks, plan->muon,
                                plan->bf16_in, plan->split, step, plan->partials, flag, stream);
    const int32_t chain = plan->split ? kNsChainSplit : kNsChainHalf;
    auto run_list = [&](const TileList &list, auto launch) {
        if (err == hipSuccess && list.n)
            err = launch(list.tiles, list.n);
    };
    for (int32_t k = 0; k < ns.steps && err == hipSuccess; ++k) {
        const bool last = k + 1 == ns.steps;
        const NsTurn turn{k % chain, {k & 1, k / chain & 1}};
        const bool begins = turn.turn == 0, ends = last || turn.turn + 1 == chain;
        run_list(plan->sym[!begins], [&](const NsTile *tiles, int32_t n) {
            return launch_ns_gram(plan->matrices, tiles, n, plan->sym_shape, plan->split, turn,
                                  stream);
        });
        run_list(plan->sym[0], [&](const NsTile *tiles, int32_t n) {
            return launch_ns_poly(plan->matrices, tiles, n, plan->sym_shape, plan->split, turn,
                                  step, stream);
        });
        auto product = [&](const NsTile *tiles, int32_t n) {
            return launch_ns_product(plan->matrices, tiles, n, plan->sym_shape, plan->split, turn,
                                     stream);
        };
        // Q = P at first, and A is not needed after the last P: then only one of the two
        if (!begins || !ends)
            run_list(begins ? plan->only_t : ends ? plan->only_q : plan->both, product);
        if (!ends)
            run_list(plan->next_gram, product);
        run_list(plan->update[!ends], [&](const NsTile *tiles, int32_t n) {
            return launch_ns_update(plan->matrices, tiles, n, plan->update_shape, plan->split,
                                    turn, last, plan->kind, step, flag, stream);
        });
    }
    if (err != hipSuccess)
        return fail_hip(err, "kernel launch");
    return LAMB_OK;
}

lamb_status check_side(int32_t i, int64_t rows, int64_t cols) {
    if (rows < 1 || rows > kMaxSide || cols < 1 || cols > kMaxSide)
        return fail(LAMB_EINVAL, "matrix %d is %lld x %lld, need 1 to 2^20 each", i,
                    static_cast<long long>(rows), static_cast<long long>(cols));
    return LAMB_OK;
}

lamb_status finish(lamb_ns_plan *plan, std::vector<NsMatrix> &matrices, lamb_ns_plan **out) {
    const lamb_status st = guarded([&] { return build(plan, matrices); });
    if (st != LAMB_OK) {
        if (plan->block)
            (void)hipFree(plan->block);
        if (plan->order.done)
            (void)hipEventDestroy(plan->order.done);
        delete plan;
        return st;
    }
    *out = plan;
    return LAMB_OK;
}

lamb_status check_precision(int32_t precision) {
    if (precision != LAMB_NS_HALF && precision != LAMB_NS_SPLIT)
        return fail(LAMB_EINVAL, "unknown precision %d", precision);
    return LAMB_OK;
}

}  // namespace

extern "C" {

lamb_status lamb_ns_params_init(lamb_ns_params *params) {
    if (!params)
        return fail(LAMB_ENULL, "params must not be NULL");
    *params = lamb_ns_params{5, 3.4445f, -4.7750f, 2.0315f, 1e-7f, 0};
    return LAMB_OK;
}

lamb_status lamb_muon_hparams_init(lamb_muon_hparams *hp) {
    if (!hp)
        return fail(LAMB_ENULL, "hparams must not be NULL");
    *hp = lamb_muon_hparams{};
    (void)lamb_ns_params_init(&hp->ns);
    hp->lr = 1e-3f;
    hp->momentum = 0.95;
    hp->grad_scale = 1.0f;
    hp->nesterov = 1;
    hp->scale = LAMB_MUON_RMS;
    return LAMB_OK;
}

lamb_status lamb_ortho_plan_create(const lamb_matrix *matrices, int32_t n, int32_t in_dtype,
                                   int32_t out_dtype, int32_t precision, lamb_ns_plan **out) {
    if (!out)
        return fail(LAMB_ENULL, "out must not be NULL");
    *out = nullptr;
    if (!matrices)
        return fail(LAMB_ENULL, "matrices must not be NULL");
    if (n < 1)
        return fail(LAMB_EINVAL, "n = %d, need >= 1", n);
    if (!is_float(in_dtype) || !is_float(out_dtype))
        return fail(LAMB_EINVAL, "matrices are float32 or bfloat16");
    lamb_status st = check_precision(precision);
    if (st != LAMB_OK)
        return st;
    return guarded([&]() -> lamb_status {
        const int64_t in_size = size_of(in_dtype), out_size = size_of(out_dtype);
        std::vector<NsMatrix> list;
        std::vector<Span> spans;
        for (int32_t i = 0; i < n; ++i) {
            const lamb_matrix &t = matrices[i];
            if (!t.in || !t.out)
                return fail(LAMB_ENULL, "matrix %d: in and out must not be NULL", i);
            lamb_status s = check_side(i, t.rows, t.cols);
            if (s != LAMB_OK)
                return s;
            if (t.in_stride < t.cols || t.out_stride < t.cols || t.in_stride > kMaxStride ||
                t.out_stride > kMaxStride)
                return fail(LAMB_EINVAL,
                            "matrix %d: a row stride is below its %lld columns, or above 2^36", i,
                            static_cast<long long>(t.cols));
            if (!aligned_to(t.in, uintptr_t(in_size)) || !aligned_to(t.out, uintptr_t(out_size)))
                return fail(LAMB_EALIGN, "matrix %d: a pointer is not aligned to its elements", i);
            const bool in_place =
                t.in == t.out && in_dtype == out_dtype && t.in_stride == t.out_stride;
            if (!in_place)
                spans.push_back(
                    span_of_rows(t.in, t.rows, t.in_stride, t.cols, in_size, false, i, "in"));
            spans.push_back(
                span_of_rows(t.out, t.rows, t.out_stride, t.cols, out_size, true, i, "out"));
            NsMatrix m{};
            m.in = t.in;
            m.out = t.out;
            m.rows = int32_t(t.rows);
            m.cols = int32_t(t.cols);
            m.in_stride = t.in_stride;
            m.out_stride = t.out_stride;
            m.vector = aligned_to(t.in, 16) && aligned_to(t.out, 16) &&
                       t.in_stride * in_size % 16 == 0 && t.out_stride * out_size % 16 == 0;
            list.push_back(m);
        }
        lamb_status s = check_spans(spans.data(), spans.size());
        if (s != LAMB_OK)
            return s;
        lamb_ns_plan *plan = new lamb_ns_plan;
        plan->bf16_in = in_dtype == LAMB_DTYPE_BF16;
        plan->split = precision == LAMB_NS_SPLIT;
        plan->kind = out_dtype == LAMB_DTYPE_BF16 ? kNsBf16Out : kNsF32Out;
        return finish(plan, list, out);
    });
}

lamb_status lamb_muon_plan_create(const lamb_muon_tensor *tensors, int32_t n, int32_t g_dtype,
                                  int32_t precision, lamb_ns_plan **out) {
    if (!out)
        return fail(LAMB_ENULL, "out must not be NULL");
    *out = nullptr;
    if (!tensors)
        return fail(LAMB_ENULL, "tensors must not be NULL");
    if (n < 1)
        return fail(LAMB_EINVAL, "n = %d, need >= 1", n);
    if (!is_float(g_dtype))
        return fail(LAMB_EINVAL, "gradients are float32 or bfloat16");
    lamb_status st = check_precision(precision);
    if (st != LAMB_OK)
        return st;
    return guarded([&]() -> lamb_status {
        std::vector<NsMatrix> list;
        std::vector<Span> spans;
        for (int32_t i = 0; i < n; ++i) {
            const lamb_muon_tensor &t = tensors[i];
            if (!t.x || !t.g || !t.m)
                return fail(LAMB_ENULL, "matrix %d: x, g and m must not be NULL", i);
            lamb_status s = check_side(i, t.rows, t.cols);
            if (s != LAMB_OK)
                return s;
            if (t.wd != 0 && t.wd != 1)
                return fail(LAMB_EINVAL, "matrix %d: wd must be 0 or 1", i);
            if (t.reserved != 0)
                return fail(LAMB_EINVAL, "matrix %d: reserved field must be 0", i);
            if (!aligned_to(t.x, 16) || !aligned_to(t.g, 16) || !aligned_to(t.m, 16))
                return fail(LAMB_EALIGN, "matrix %d: every buffer must be 16-byte aligned", i);
            const uint64_t numel = uint64_t(t.rows) * uint64_t(t.cols);
            spans.push_back(span_of(t.x, numel * 4, true, i, "x"));
            spans.push_back(span_of(t.g, numel * uint64_t(size_of(g_dtype)), false, i,
                                    "g"));
            spans.push_back(span_of(t.m, numel * 4, true, i, "m"));
            NsMatrix m{};
            m.in = t.g;
            m.out = t.x;
            m.m = t.m;
            m.rows = int32_t(t.rows);
            m.cols = int32_t(t.cols);
            m.in_stride = m.out_stride = t.cols;
            m.vector = t.cols % 8 == 0;
            m.wd = t.wd;
            list.push_back(m);
        }
        lamb_status s = check_spans(spans.data(), spans.size());
        if (s != LAMB_OK)
            return s;
        lamb_ns_plan *plan = new lamb_ns_plan;
        plan->muon = true;
        plan->bf16_in = g_dtype == LAMB_DTYPE_BF16;
        plan->split = precision == LAMB_NS_SPLIT;
        plan->kind = kNsMuon;
        return finish(plan, list, out);
    });
}

lamb_status lamb_orthogonalize(lamb_ns_plan *plan, const lamb_ns_params *params, void *stream) {
    if (!plan || !params)
        return fail(LAMB_ENULL, "plan and params must not be NULL");
    if (plan->muon)
        return fail(LAMB_EPLAN, "the plan was created for lamb_muon_step");
    lamb_status st = check_params(*params);
    if (st != LAMB_OK)
        return st;
    DeviceScope scope(plan->device);
    hipStream_t on = static_cast<hipStream_t>(stream);
    return ordered(plan->order, on,
                   [&] { return run(plan, *params, NsStep{}, nullptr, nullptr, on); });
}

lamb_status lamb_muon_check(const lamb_ns_plan *plan, const lamb_muon_hparams *hp) {
    if (!plan || !hp)
        return fail(LAMB_ENULL, "plan and hparams must not be NULL");
    if (!plan->muon)
        return fail(LAMB_EPLAN, "the plan was created for lamb_orthogonalize");
    lamb_status st = check_params(hp->ns);
    if (st != LAMB_OK)
        return st;
    if (!std::isfinite(hp->lr) || hp->lr < 0.0f)
        return fail(LAMB_EINVAL, "lr = %g, need finite and >= 0", double(hp->lr));
    if (!(hp->momentum >= 0.0 && hp->momentum < 1.0))
        return fail(LAMB_EINVAL, "momentum = %g outside [0, 1)", hp->momentum);
    if (!std::isfinite(hp->weight_decay) || hp->weight_decay < 0.0f)
        return fail(LAMB_EINVAL, "weight_decay = %g, need finite and >= 0",
                    double(hp->weight_decay));
    if (!std::isfinite(hp->grad_scale) || hp->grad_scale <= 0.0f)
        return fail(LAMB_EINVAL, "grad_scale = %g, need finite and > 0", double(hp->grad_scale));
    if ((hp->nesterov | hp->skip_nonfinite) & ~1)
        return fail(LAMB_EINVAL, "nesterov and skip_nonfinite must be 0 or 1");
    if (hp->scale < LAMB_MUON_RMS || hp->scale > LAMB_MUON_UNIT)
        return fail(LAMB_EINVAL, "unknown scale %d", hp->scale);
    if (hp->reserved != 0)
        return fail(LAMB_EINVAL, "hparams.reserved must be 0");
    return LAMB_OK;
}

lamb_status lamb_muon_step(lamb_ns_plan *plan, const lamb_muon_hparams *hp, void *stream_in,
                           int32_t *nonfinite_out) {
    const lamb_status st = lamb_muon_check(plan, hp);
    if (st != LAMB_OK)
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    DeviceScope scope(plan->device);
    NsStep step{};
    step.momentum = hp->momentum;
    step.from_grad = (1.0 - hp->momentum) * double(hp->grad_scale);
    step.decay = float(1.0 - double(hp->lr) * double(hp->weight_decay));
    step.lr = hp->lr;
    step.nesterov = hp->nesterov;
    step.scale = hp->scale;
    return ordered(plan->order, stream, [&] {
        uint32_t *flag = nullptr;
        if (hp->skip_nonfinite) {
            const hipError_t err =
                launch_ns_check(plan->matrices, plan->block_matrix, plan->blocks, plan->bf16_in,
                                hp->grad_scale, plan->flag, stream);
            if (err != hipSuccess)
                return fail_hip(err, "kernel launch");
            flag = plan->flag;
        }
        return run(plan, hp->ns, step, flag, nonfinite_out, stream);
    });
}

lamb_status lamb_ns_plan_destroy(lamb_ns_plan *plan) {
    if (!plan)
        return LAMB_OK;
    DeviceScope scope(plan->device);
    hipError_t err = hipFree(plan->block);  // waits for what still uses it
    const hipError_t event = hipEventDestroy(plan->order.done);
    if (err == hipSuccess)
        err = event;
    delete plan;
    if (err != hipSuccess)
        return fail_hip(err, "hipFree, hipEventDestroy");
    return LAMB_OK;
}

}  // extern "C"
