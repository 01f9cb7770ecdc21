// Prints the form that each product read from standard input takes, by the library's own rule: "int8 m n k", or "grouped" or
// "turned" with rows, groups and outputs.
#include <cstdio>
#include <cstring>

#include "grouped_plan.h"

int main() {
    char op[16];
    long long a, b, c;
    while (std::scanf("%15s %lld %lld %lld", op, &a, &b, &c) == 4) {
        if (!std::strcmp(op, "int8")) {
            using namespace product_plan;
            if (a <= kDotRows) {
                std::puts("dot");
                continue;
            }
            const Plan p = plan_product<kInt8, kSums>(a, b, up(c, 16));
            std::printf("tile%d %s %s%s\n", p.tile, p.parts > 1 ? "split" : "whole", b % 8 ? "values" : "lines",
                        p.parts > 1 && b > 1024 ? " joined in pieces" : "");
        } else {
            const grouped_plan::GroupedPlan p = grouped_plan::plan_grouped(a, b, c, !std::strcmp(op, "turned"));
            std::printf("%d x %d by %d\n", p.height, p.width, p.threads);
        }
    }
    return 0;
}
