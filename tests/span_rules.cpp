// The overlap check of the operators' entry points (ops_host.h) against every byte of
// small layouts: what is let through shares no written byte, and of operands with one
// stride, or without rows of their own, all that share none are let through.
#include <stdarg.h>
#include <stdio.h>

#include <random>

#include "ops_host.h"

namespace lamb_mi355x {
lamb_status fail(lamb_status status, const char *, ...) { return status; }
}  // namespace lamb_mi355x

using namespace lamb_mi355x;

int main() {
    std::mt19937 rng(1);
    auto pick = [&](int low, int high) { return int(rng() % unsigned(high - low + 1)) + low; };
    int let_through = 0, refused = 0, spared = 0;
    for (int round = 0; round < 400000; ++round) {
        const bool one_stride = round % 2;
        const int common = pick(2, 9), n = pick(2, 4);
        Span spans[4];
        int readers[400] = {}, writers[400] = {};
        bool shared = false, runs = false;
        for (int i = 0; i < n; ++i) {
            const int size = pick(0, 1) ? 2 : 4;
            const int stride = one_stride ? common * 4 / size : pick(1, 9);
            const int rows = pick(0, 5), cols = pick(1, stride < 4 ? stride : pick(1, stride));
            const int at = 4 * pick(0, one_stride ? 2 * common : 30);
            const bool written = pick(0, 2) > 0;
            spans[i] = span_of_rows(reinterpret_cast<const void *>(uintptr_t(at + 4096)), rows,
                                    stride, cols, size, written, i, "span");
            // a run without rows of its own that reaches over another's rows is refused by
            // its ends, rightly: the rows lie in it
            runs |= rows == 1;
            for (int r = 0; r < rows; ++r)
                for (int b = 0; b < cols * size; ++b) {
                    const int byte = at + r * stride * size + b;
                    if (byte >= 400)
                        return printf("layout too large\n"), 1;
                    (written ? writers : readers)[byte] += 1;
                }
        }
        for (int b = 0; b < 400; ++b) shared |= writers[b] > 1 || (writers[b] && readers[b]);
        const lamb_status st = check_spans(spans, size_t(n));
        if (st == LAMB_OK && shared)
            return printf("round %d: shared bytes let through\n", round), 1;
        if (st != LAMB_OK && !shared && one_stride && !runs)
            return printf("round %d: operands of one stride refused\n", round), 1;
        spared += st != LAMB_OK && !shared;
        (st == LAMB_OK ? let_through : refused) += 1;
    }
    if (let_through < 10000 || refused < 10000)
        return printf("%d let through, %d refused\n", let_through, refused), 1;
    printf("all checks passed (%d let through, %d refused, %d of them by their ends)\n",
           let_through, refused, spared);
    return 0;
}
