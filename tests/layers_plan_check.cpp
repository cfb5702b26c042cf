// What the launch rules of the layers and losses choose, for sizes read from standard input (built and run by tests/test_layers_plan.py).  A line is
//     linear bytes learners tokens in out cus | grad bytes learners tokens in out cus | logprobs bytes rows columns k 0 cus | distill bytes rows columns gradient 0 cus
// and its answer one line of words.
#include <cstdio>
#include <cstring>

#include "psgd_layers_plan.h"

using namespace psgd;

static void product(const char* name, const Plan& p, int64_t k, int bytes) {
    std::printf(" %s=%dx%d%s%s", name, p.rows, p.cols, p.split > 1 ? "/parts" : "", short_k(k, bytes) ? "/short" : "");
}

int main() {
    char what[16];
    int bytes;
    long long a, b, c, d, cus;
    while (std::scanf("%15s %d %lld %lld %lld %lld %lld", what, &bytes, &a, &b, &c, &d, &cus) == 7) {
        std::printf("%s", what);
        if (!std::strcmp(what, "linear")) {              // learners, tokens, in, out
            if (b <= most_few((int)a, d, bytes, (int)cus))
                std::printf(" few=%d/%d", b <= 1 ? 1 : b <= 2 ? 2 : b <= 4 ? 4 : 8, four_outputs((int)a, d, (int)cus) && b <= 4 ? 4 : 1);
            else
                product("y", forward_plan((int)a, b, d, c, bytes, (int)cus), c, bytes);
        } else if (!std::strcmp(what, "grad")) {
            const GradPlan g = grad_plan((int)a, b, c, d, bytes, (int)cus, true, true);
            if (g.pair) {
                std::printf(" pair=%d", g.dx.rows);
            } else {
                product("dx", g.dx, d, bytes);
                if (g.few) std::printf(" dwfew=%d/%d", b <= 2 ? 2 : b <= 4 ? 4 : b <= 8 ? 8 : 16, g.few_rows);
                else product("dw", g.dw, b, bytes);
            }
        } else {
            const int64_t groups = parts_of(b, 16 / bytes);
            if (!std::strcmp(what, "logprobs")) {        // rows, columns, k, 0
                const int lanes = lanes_of_row(a, groups, (int)c, (int)cus);
                std::printf(" lanes=%d batches=%s kept=%d", lanes, groups > (int64_t)lanes * kUnroll ? "several" : "one", batches_kept(groups, lanes) > 0);
            } else {                                     // rows, columns, gradient, 0
                const DistillHold h = distill_hold(a, groups, c != 0, (int)cus);
                std::printf(" lanes=%d held=%d", h.lanes, h.held);
            }
        }
        std::printf("\n");
    }
}
