// Reads lines "kind type n tokens width channels" (kind 0: the product, 1: dX,
// 2: dW) and prints "tile split blocks workspace" of each product's plan.
#include <cstdio>

#include "../../paper_2110_04175_amd/csrc/layer_plan.hpp"

int main() {
    int kind, type;
    long long n, tokens, width, channels;
    while (std::scanf("%d %d %lld %lld %lld %lld", &kind, &type, &n, &tokens, &width, &channels) == 6) {
        const layer_plan::Plan p = kind == 0   ? layer_plan::plan_linear((int32_t)n, tokens, width, channels)
                                   : kind == 1 ? layer_plan::plan_grad(type, n, tokens, width, channels)
                                               : layer_plan::plan_grad(type, n, channels, width, tokens);
        std::printf("%d %d %lld %zu\n", p.tile, p.split, (long long)p.blocks, p.workspace);
    }
}
