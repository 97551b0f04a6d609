/*
 * Sanitizer driver for the host code of the attention to other states (CPU only): linked
 * with AddressSanitizer / UndefinedBehaviorSanitizer builds of cross_api.hip, cross_fwd.hip
 * and cross_bwd.hip, it asks for workspaces over small, odd and extreme sizes (which runs the
 * plans of the launches) and makes calls that are refused before any HIP call.
 */
#include <stdio.h>

#include "fibattn.h"

static int bad = 0;
#define EXPECT(cond)                                                   \
    do {                                                               \
        if (!(cond)) { fprintf(stderr, "line %d: %s\n", __LINE__, #cond); bad = 1; } \
    } while (0)

int main() {
    const int sizes[] = {1, 2, 7, 31, 32, 33, 127, 129, 512, 513, 1000, 4097, 65535, 1 << 20, 1 << 30};
    const int heads[][2] = {{1, 1}, {8, 1}, {8, 2}, {7, 7}, {64, 8}, {65535, 1}};
    for (int S : sizes)
        for (int T : sizes)
            for (int B : {1, 3, 64, 1024})
                for (const auto &h : heads)
                    for (int D : {32, 64, 128}) {
                        const bool ok = (long long)B * h[0] <= 65535 && (long long)B * h[0] * T <= 1 << 30;
                        const size_t own = fibattn_cross_backward_workspace_bytes(B, B, h[0], h[1], T, S, D);
                        const size_t shared = fibattn_cross_backward_workspace_bytes(B, 1, h[0], h[1], T, S, D);
                        const size_t pre = fibattn_prefix_workspace_bytes(B, h[0], h[1], T, S, T, D);
                        EXPECT(ok ? own > 0 && shared > 0 && pre > 0 : !own && !shared && !pre);
                        EXPECT(ok || !fibattn_cross_workspace_bytes(B, B, h[0], h[1], T, S, D));
                        // partial results stay a small multiple of what they are parts of
                        const double rows = (double)B * h[0] * T;
                        EXPECT(!ok || (double)pre <= 129 * (rows * (D + 1) * 4 + 512));
                    }
    EXPECT(fibattn_cross_workspace_bytes(-1, -1, 4, 4, 8, 8, 64) == 0);
    EXPECT(fibattn_cross_workspace_bytes(0x7fffffff, 1, 0x7fffffff, 1, 0x7fffffff, 0x7fffffff, 64) == 0);
    void *p = (void *)4096;
    float *f = (float *)4096;
    const fibattn_layout_t odd[8] = {{3, 8, 8}, {0, 0, 0}, {0, 0, 0}, {0, 0, 0}, {0, 0, 0}, {0, 0, 0}, {0, 0, 0}, {0, 0, 0}};
    EXPECT(fibattn_cross_forward(p, p, p, p, f, nullptr, p, 1u << 30, odd, 1, 1, 4, 2, 8, 8, 64, FIBATTN_BF16, nullptr) ==
           FIBATTN_ERR_INVALID_ARG);
    EXPECT(fibattn_cross_backward(p, p, p, p, f, p, p, p, p, nullptr, p, 0, nullptr, 1, 1, 4, 2, 8, 8, 64, FIBATTN_FP32,
                                  nullptr) == FIBATTN_ERR_WORKSPACE);
    EXPECT(fibattn_prefix_forward(p, p, p, p, p, nullptr, f, nullptr, p, 1u << 30, nullptr, 1, 4, 2, 8, 8, 8, 64,
                                  FIBATTN_FP32, nullptr) == FIBATTN_ERR_INVALID_ARG);
    EXPECT(fibattn_join(p, f, p, f, p, f, nullptr, 1, 4, 8, 65, FIBATTN_FP32, nullptr) == FIBATTN_ERR_UNSUPPORTED);
    EXPECT(fibattn_join(p, f, p, f, p, f, nullptr, 1, 4, 8, 64, (fibattn_dtype_t)9, nullptr) == FIBATTN_ERR_INVALID_ARG);
    printf(bad ? "FAILED\n" : "OK\n");
    return bad;
}
