// Answers, for sizes on standard input, what the launch rules of the attention blocks choose (csrc/psgd_attention_plan.h).
#include <cstdio>
#include <cstring>

#include "psgd_attention_plan.h"

int main() {
    char kind[16];
    while (std::scanf("%15s", kind) == 1) {
        long long a[9];
        if (!std::strcmp(kind, "grad")) {          // bytes heads kv head window sinks sequences n t
            for (auto& x : a)
                if (std::scanf("%lld", &x) != 1) return 1;
            const psgd::KeyParts p = psgd::key_parts((int)a[1], (int)a[2], (int)a[3], (int)a[0], a[4], a[5], (int)a[6], (int)a[7], a[8]);
            std::printf("%d %d %d %d %d %lld %lld %zu %zu\n", p.most, p.steps, p.first_tiles, p.first_most, p.first_steps, (long long)p.slots, (long long)p.first_slots,
                        p.slot_bytes, p.bytes(a[7] * a[2]));
        } else if (!std::strcmp(kind, "step")) {   // bytes units most_keys head
            for (int i = 0; i < 4; ++i)
                if (std::scanf("%lld", &a[i]) != 1) return 1;
            std::printf("%d\n", psgd::step_parts(a[1], a[2], (int)a[3], (int)a[0]));
        } else if (!std::strcmp(kind, "forward")) {   // bytes head t heads
            for (int i = 0; i < 4; ++i)
                if (std::scanf("%lld", &a[i]) != 1) return 1;
            std::printf("%d\n", psgd::forward_blocks(psgd::held_head((int)a[1]), (int)a[0], a[2], a[3]));
        } else if (!std::strcmp(kind, "shape")) {  // bytes head
            for (int i = 0; i < 2; ++i)
                if (std::scanf("%lld", &a[i]) != 1) return 1;
            const int held = psgd::held_head((int)a[1]), bytes = (int)a[0];
            std::printf("%d %d %d %d %d %d\n", held, psgd::in_lds(held), psgd::own_rows(held, bytes), psgd::walked_rows(held, bytes), psgd::query_rows(held, bytes),
                        psgd::step_waves(held, bytes));
        } else {
            return 1;
        }
    }
    return 0;
}
