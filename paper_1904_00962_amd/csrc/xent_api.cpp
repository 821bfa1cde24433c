// Host side of the cross entropy of include/lamb_ops.h: validation, the workspace's
// layout and the launches of a call.
#include <math.h>

#include "ops_host.h"
#include "xent_internal.h"

using namespace lamb_mi355x;

namespace {

constexpr int64_t kMaxReadStride = int64_t(1) << 21;  // a tile's rows within 32-bit offsets
// A piece of the vocabulary's softmax: written once and read twice, so kept within
// the 256 MiB last-level cache, unless so many tokens leave it fewer than kPieceAlign words.
constexpr int64_t kPieceBytes = int64_t(160) << 20;
constexpr int64_t kPieceAlign = 256;  // half of it where Q is in two parts

lamb_status check(const lamb_xent *x) {
    if (!x)
        return fail(LAMB_ENULL, "xent must not be NULL");
    if (x->reserved != 0)
        return fail(LAMB_EINVAL, "xent.reserved must be 0");
    if (x->tokens < 0 || x->tokens > kMaxTokens || x->vocab < 1 || x->vocab > kMaxVocab ||
        x->dim < 1 || x->dim > kMaxDim)
        return fail(LAMB_EINVAL,
                    "tokens %lld, vocab %lld, dim %lld: need 0 to 2^24, 1 to 2^24, 1 to 2^16",
                    (long long)x->tokens, (long long)x->vocab, (long long)x->dim);
    if (!is_id(x->target_dtype))
        return fail(LAMB_EINVAL, "targets are int32 or int64");
    if (!x->table || (x->tokens && (!x->hidden || !x->targets)))
        return fail(LAMB_ENULL, "hidden, table and targets must not be NULL");
    if (x->hidden_stride < x->dim || x->table_stride < x->dim || x->hidden_stride > kMaxStride ||
        x->table_stride > kMaxStride)
        return fail(LAMB_EINVAL, "a row stride is below dim, or above 2^36");
    if (!aligned_to(x->hidden, 2) || !aligned_to(x->table, 2) ||
        !aligned_to(x->targets, uintptr_t(size_of(x->target_dtype))))
        return fail(LAMB_EALIGN, "a pointer is not aligned to its elements");
    return LAMB_OK;
}

bool in_place(const void *p, int64_t stride, int64_t dim) {
    return dim % 8 == 0 && stride % 8 == 0 && stride <= kMaxReadStride && aligned_to(p, 16);
}

int64_t count_tiles(int64_t rows, int64_t cols, int shape) {
    const int64_t t = xent_tile(shape);
    return (rows + t - 1) / t * ((cols + t - 1) / t);
}

// The tile shape of a product of `rows` x `cols` over `depth`, the parts that `depth`
// is cut in (at most `most`), and the time, by the least estimate: rounds of workgroups
// over the CUs times a tile's time. Microseconds, measured on one GPU: a tile's fixed
// part, and per 1024 of depth where all CUs work (two of the smaller tiles share one).
struct Product {
    int shape = 0;
    int32_t parts = 1;
    double time = 1e300;
};

Product pick(int64_t rows, int64_t cols, int64_t depth, int64_t most) {
    constexpr double kFixed[3] = {2.0, 4.0, 15.0}, kDeep[3] = {8.4, 18.0, 23.0};
    constexpr int64_t kSlots[3] = {512, 512, 256};
    constexpr double kBytesPerUs = 5e6;
    Product best;
    for (int shape = kXentTiny; shape <= kXentLarge; ++shape) {
        const int64_t tiles = std::max<int64_t>(1, count_tiles(rows, cols, shape));
        // more than two rounds of parts never pay
        const int64_t limit = std::min<int64_t>({most, 32, 2 * kSlots[shape] / tiles + 1});
        for (int64_t parts = 1; parts <= limit; ++parts) {
            const int64_t rounds = (tiles * parts + kSlots[shape] - 1) / kSlots[shape];
            // a part more writes and reads rows x cols of fp32 once more
            const double time = double(rounds) * (kFixed[shape] + double(depth) / double(parts) /
                                                                      1024.0 * kDeep[shape]) +
                                double(parts - 1) * double(rows) * double(cols) * 8.0 / kBytesPerUs;
            if (time < best.time)
                best = Product{shape, int32_t(parts), time};
        }
    }
    return best;
}

// The backward's pieces of the vocabulary, and the shapes of their products.
struct Pieces {
    int64_t size = 0;
    int probs_shape = 0, hidden_shape = 0, table_shape = 0;
    int32_t splits = 1;  // workgroups that share the sum of a tile of dH
    double time = 1e300;
};

// Equal pieces whose Q, in `q_parts` parts, has at most kPieceBytes: of the next few counts,
// the one whose products fill their last rounds of workgroups best.
Pieces pick_pieces(const lamb_xent &x, int32_t q_parts) {
    const int64_t rows = x.tokens ? x.tokens : 1, align = kPieceAlign / q_parts;
    const int64_t most =
        std::max<int64_t>(align, kPieceBytes / 2 / q_parts / rows / align * align);
    const int64_t least = (x.vocab + most - 1) / most;
    Pieces best;
    for (int64_t count = least; count < least + 4; ++count) {
        const int64_t size =
            std::min(round_up((x.vocab + count - 1) / count, align), round_up(x.vocab, 8));
        const Product probs = pick(x.tokens, size, x.dim, 1);
        const Product table = pick(size, x.dim, q_parts * x.tokens, 1);
        // few rows: the piece's columns are split over workgroups, 256 each at least
        const Product hidden = pick(x.tokens, x.dim, size, std::max<int64_t>(1, size / 256));
        const double time = double((x.vocab + size - 1) / size) *
                            (probs.time + table.time + hidden.time);
        if (time < best.time)
            best = Pieces{size, probs.shape, hidden.shape, table.shape, hidden.parts, time};
    }
    return best;
}

struct Layout {
    int64_t ld = 0;
    bool copy_table = false;
    int logits_shape = 0;
    int32_t parts = 0;
    Pieces pieces[2];  // Q in one part, and in two
    // offsets, and the end
    size_t kept = 0, source = 0, target = 0, packed = 0, table = 0, parts_at = 0, at_target = 0,
           probs = 0, partial = 0, table_sum = 0, bytes = 0;
};

Layout layout_of(const lamb_xent &x, bool backward) {
    Layout l;
    l.ld = round_up(x.dim, 8);
    l.copy_table = !in_place(x.table, x.table_stride, x.dim);
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t start = at;
        at += size_t(round_up(bytes, 256));
        return start;
    };
    l.kept = take(4);
    l.source = take(4 * x.tokens);
    l.target = take(4 * x.tokens);
    l.packed = take(2 * x.tokens * l.ld);
    l.table = take(l.copy_table ? 2 * x.vocab * l.ld : 0);
    if (!backward) {
        l.logits_shape = pick(x.tokens, x.vocab, x.dim, 1).shape;
        const int32_t tile = xent_tile(l.logits_shape);
        l.parts = int32_t((x.vocab + tile - 1) / tile);
        l.parts_at = take(int64_t(l.parts) * x.tokens * 8);
        l.at_target = take(4 * x.tokens);
        l.bytes = at;
        return l;
    }
    int64_t probs = 0;
    int32_t splits = 1;
    for (int32_t k = 0; k < 2; ++k) {
        l.pieces[k] = pick_pieces(x, k + 1);
        probs = std::max(probs, (k + 1) * 2 * x.tokens * l.pieces[k].size);
        splits = std::max(splits, l.pieces[k].splits);
    }
    l.probs = take(probs);
    l.partial = take(int64_t(splits) * x.tokens * l.ld * 4);
    l.table_sum = take(x.tokens > kChainTokens
                           ? std::max(l.pieces[0].size, l.pieces[1].size) * l.ld * 4
                           : 0);
    l.bytes = at;
    return l;
}

// The packed rows and the table as the kernels read them.
lamb_status begin(const lamb_xent &x, const Layout &l, char *work, float *loss, float *lse,
                  void *grad_hidden, int64_t grad_stride, XentArgs *args, hipStream_t stream) {
    XentPack pack{};
    pack.hidden = static_cast<const uint16_t *>(x.hidden);
    pack.stride = x.hidden_stride;
    pack.targets = x.targets;
    pack.wide = x.target_dtype == LAMB_DTYPE_I64;
    pack.vector = aligned_to(x.hidden, 16) && x.hidden_stride % 8 == 0;
    pack.ignore = x.ignore_index;
    pack.dim = int32_t(x.dim);
    pack.ld = int32_t(l.ld);
    pack.vocab = int32_t(x.vocab);
    pack.tokens = int32_t(x.tokens);
    pack.rounds = pack_rounds(x.tokens);
    pack.packed = reinterpret_cast<uint16_t *>(work + l.packed);
    pack.kept = reinterpret_cast<int32_t *>(work + l.kept);
    pack.source = reinterpret_cast<int32_t *>(work + l.source);
    pack.target = reinterpret_cast<int32_t *>(work + l.target);
    pack.loss = loss;
    pack.lse = lse;
    pack.grad_hidden = static_cast<uint16_t *>(grad_hidden);
    pack.grad_stride = grad_stride;
    hipError_t err = launch_xent_pack(pack, stream);
    *args = XentArgs{};
    args->hidden = pack.packed;
    args->ld = l.ld;
    args->table = static_cast<const uint16_t *>(x.table);
    args->table_ld = x.table_stride;
    if (l.copy_table) {
        uint16_t *copy = reinterpret_cast<uint16_t *>(work + l.table);
        if (err == hipSuccess)
            err = launch_xent_copy(args->table, x.table_stride, copy, int32_t(x.dim),
                                   int32_t(l.ld), x.vocab, stream);
        args->table = copy;
        args->table_ld = l.ld;
    }
    args->dim = int32_t(x.dim);
    args->vocab = int32_t(x.vocab);
    args->tokens = int32_t(x.tokens);
    args->kept = pack.kept;
    args->source = pack.source;
    args->target = pack.target;
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

}  // namespace

extern "C" {

lamb_status lamb_xent_workspace(const lamb_xent *xent, size_t *forward_bytes,
                                size_t *backward_bytes) {
    const lamb_status st = check(xent);
    if (st != LAMB_OK)
        return st;
    if (forward_bytes)
        *forward_bytes = layout_of(*xent, false).bytes;
    if (backward_bytes)
        *backward_bytes = layout_of(*xent, true).bytes;
    return LAMB_OK;
}

lamb_status lamb_xent_forward(const lamb_xent *xent, float *loss, float *lse, float *mean,
                              void *workspace, size_t workspace_bytes, void *stream_in) {
    lamb_status st = check(xent);
    if (st != LAMB_OK)
        return st;
    const lamb_xent &x = *xent;
    if (x.tokens && (!loss || !lse))
        return fail(LAMB_ENULL, "loss and lse must not be NULL");
    if (!aligned_to(loss, 4) || !aligned_to(lse, 4) || !aligned_to(mean, 4))
        return fail(LAMB_EALIGN, "a pointer is not aligned to its elements");
    const Layout l = layout_of(x, false);
    st = check_workspace(workspace, workspace_bytes, l.bytes);
    if (st != LAMB_OK)
        return st;
    const int64_t id = size_of(x.target_dtype);
    Span spans[] = {
        span_of_rows(x.hidden, x.tokens, x.hidden_stride, x.dim, 2, false, 0, "hidden"),
        span_of_rows(x.table, x.vocab, x.table_stride, x.dim, 2, false, 0, "table"),
        span_of(x.targets, uint64_t(x.tokens * id), false, 0, "targets"),
        span_of(loss, uint64_t(x.tokens) * 4, true, 0, "loss"),
        span_of(lse, uint64_t(x.tokens) * 4, true, 0, "lse"),
        span_of(mean, mean ? 4 : 0, true, 0, "mean"),
        span_of(workspace, l.bytes, true, 0, "workspace")};
    st = check_spans(spans, sizeof spans / sizeof spans[0]);
    if (st != LAMB_OK)
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    char *work = static_cast<char *>(workspace);
    XentArgs args;
    st = begin(x, l, work, loss, lse, nullptr, 0, &args, stream);
    if (st != LAMB_OK)
        return st;
    hipError_t err = hipSuccess;
    const bool few = x.tokens > 0 && x.tokens <= kReduceTokens;  // one workgroup reduces
    if (x.tokens) {
        float2 *parts = reinterpret_cast<float2 *>(work + l.parts_at);
        float *at_target = reinterpret_cast<float *>(work + l.at_target);
        err = launch_xent_logits(args, l.logits_shape, parts, at_target, stream);
        if (err == hipSuccess)
            err = launch_xent_reduce(args, l.parts, parts, at_target, loss, lse,
                                     few ? mean : nullptr, stream);
    }
    if (err == hipSuccess && mean && !few)
        err = launch_xent_mean(loss, args.tokens, args.kept, mean, stream);
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

lamb_status lamb_xent_backward(const lamb_xent *xent, const float *lse,
                               const lamb_xent_grads *grads, void *workspace,
                               size_t workspace_bytes, void *stream_in) {
    lamb_status st = check(xent);
    if (st != LAMB_OK)
        return st;
    const lamb_xent &x = *xent;
    if (!grads || (x.tokens && !lse))
        return fail(LAMB_ENULL, "lse and grads must not be NULL");
    const lamb_xent_grads &g = *grads;
    if ((g.add_table | g.mean) & ~1)
        return fail(LAMB_EINVAL, "grads.add_table and grads.mean must be 0 or 1");
    if (!std::isfinite(g.grad_scale))
        return fail(LAMB_EINVAL, "grads.grad_scale = %g must be finite", double(g.grad_scale));
    const bool bf16 = g.grad_table_dtype == LAMB_DTYPE_BF16;
    if (g.grad_table && !is_float(g.grad_table_dtype))
        return fail(LAMB_EINVAL, "grad_table is float32 or bfloat16");
    if ((g.grad_hidden && (g.grad_hidden_stride < x.dim || g.grad_hidden_stride > kMaxStride)) ||
        (g.grad_table && (g.grad_table_stride < x.dim || g.grad_table_stride > kMaxStride)))
        return fail(LAMB_EINVAL, "a row stride is below dim, or above 2^36");
    if (!aligned_to(g.grad_loss, 4) || !aligned_to(lse, 4) || !aligned_to(g.grad_hidden, 2) ||
        !aligned_to(g.grad_table, bf16 ? 2 : 4))
        return fail(LAMB_EALIGN, "a pointer is not aligned to its elements");
    const Layout l = layout_of(x, true);
    st = check_workspace(workspace, workspace_bytes, l.bytes);
    if (st != LAMB_OK)
        return st;
    const int64_t id = size_of(x.target_dtype);
    Span spans[] = {
        span_of_rows(x.hidden, x.tokens, x.hidden_stride, x.dim, 2, false, 0, "hidden"),
        span_of_rows(x.table, x.vocab, x.table_stride, x.dim, 2, false, 0, "table"),
        span_of(x.targets, uint64_t(x.tokens * id), false, 0, "targets"),
        span_of(lse, uint64_t(x.tokens) * 4, false, 0, "lse"),
        span_of(g.grad_loss, g.grad_loss ? 4 : 0, false, 0, "grad_loss"),
        span_of_rows(g.grad_hidden, g.grad_hidden ? x.tokens : 0, g.grad_hidden_stride, x.dim, 2,
                     true, 0, "grad_hidden"),
        span_of_rows(g.grad_table, g.grad_table ? x.vocab : 0, g.grad_table_stride, x.dim,
                     bf16 ? 2 : 4, true, 0, "grad_table"),
        span_of(workspace, l.bytes, true, 0, "workspace")};
    st = check_spans(spans, sizeof spans / sizeof spans[0]);
    if (st != LAMB_OK)
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    char *work = static_cast<char *>(workspace);
    XentArgs args;
    st = begin(x, l, work, nullptr, nullptr, g.grad_hidden, g.grad_hidden_stride, &args, stream);
    if (st != LAMB_OK)
        return st;
    float *partial = reinterpret_cast<float *>(work + l.partial);
    const bool two = g.grad_table && !bf16;
    const Pieces &p = l.pieces[two];
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < x.vocab && err == hipSuccess; first += p.size) {
        XentPiece piece{};
        piece.first = int32_t(first);
        piece.count = int32_t(std::min(p.size, x.vocab - first));
        piece.ld = int32_t(round_up(piece.count, 8));
        piece.probs = reinterpret_cast<uint16_t *>(work + l.probs);
        piece.low = two ? piece.probs + x.tokens * p.size : nullptr;
        if (x.tokens)
            err = launch_xent_probs(args, p.probs_shape, piece, lse, stream);
        if (err == hipSuccess && x.tokens && g.grad_hidden)
            err = launch_xent_hidden(args, p.hidden_shape, piece, p.splits, first > 0, partial,
                                     stream);
        if (err == hipSuccess && g.grad_table)
            err = launch_xent_table(args, p.table_shape, piece, g.grad_loss, g.grad_scale, g.mean,
                                    bf16, g.add_table, g.grad_table, g.grad_table_stride,
                                    reinterpret_cast<float *>(work + l.table_sum), stream);
    }
    if (err == hipSuccess && x.tokens && g.grad_hidden)
        err = launch_xent_hidden_out(args, p.splits, partial, g.grad_loss, g.grad_scale, g.mean,
                                     static_cast<uint16_t *>(g.grad_hidden), g.grad_hidden_stride,
                                     stream);
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

}  // extern "C"
