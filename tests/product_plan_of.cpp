// Prints the form that each product read from standard input takes ("op m n k" a line), by the library's own rule.
#include <cstdio>
#include <cstring>

#include "product_plan.h"

using namespace product_plan;

template <Kind KIND, Out OUT>
void tiled(const char* form, int64_t m, int64_t n, int64_t inner) {
    const Plan p = plan_product<KIND, OUT>(m, n, inner);
    std::printf("%s tile%d %s\n", form, p.tile, p.parts > 1 ? "split" : "whole");
}

int main() {
    char op[16];
    long long m, n, k;
    while (std::scanf("%15s %lld %lld %lld", op, &m, &n, &k) == 4) {
        if (!std::strcmp(op, "linear")) {
            if (m <= kDotRows) std::puts("dot");
            else if (m <= kStreamRows) std::printf("stream%d %s\n", stream_rows_of(m), stream_parts(m, n, k) > 1 ? "split" : "whole");
            else tiled<kBf16, kSums>("sums", m, n, k);
        } else if (!std::strcmp(op, "times")) {            // estimated ones of m workgroups of each tile
            for (int t = 0; t < kTiles; ++t)
                std::printf("%.4f %.4f ", product_us<kBf16, kSums>(t, 1, m * tile_costs<kBf16>()[t].m, n, k),
                            product_us<kMx, kSums>(t, 1, m * tile_costs<kMx>()[t].m, n, k));
            std::puts("");
        } else if (!std::strcmp(op, "turns")) {            // of the stream kernel: rounds of 1024 values a workgroup
            std::printf("%lld\n", (long long)ceil_div(stream_part_values(k, stream_parts(m, n, k)), 1024));
        } else if (!std::strcmp(op, "grad") || !std::strcmp(op, "mxgrad")) {
            tiled<kBf16, kSums>("sums", m, k, n);
        } else if (!std::strcmp(op, "mx")) {
            const int64_t blocks = ceil_div(k, 32);
            if (thin(m, n, blocks)) std::puts("thin");
            else tiled<kMx, kSums>(lays_scales(m, n, blocks) ? "laid" : "mx", m, n, blocks * 32);
        } else if (!std::strcmp(op, "ffn")) {
            if (m <= kDotRows) std::puts("dot");
            else tiled<kBf16, kGate>("gate", m, n, k);
        } else if (!std::strcmp(op, "dx")) {
            tiled<kBf16, kSums>("dx", m, k, 2 * up(n, 64));
        } else if (!std::strcmp(op, "dw")) {
            tiled<kBf16, kTwoRows>("dw", 2 * n, k, m);
        } else {
            return 1;
        }
    }
    return 0;
}
