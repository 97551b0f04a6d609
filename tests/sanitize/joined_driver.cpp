/*
 * Sanitizer driver for fibattn_backward_joined (CPU only): linked with an AddressSanitizer /
 * UndefinedBehaviorSanitizer build of api.hip, it makes calls that are refused before any
 * HIP call, with host and device tables, placements and bad sizes.
 */
#include <stdio.h>

#include "fibattn.h"

static int bad = 0;
#define EXPECT(cond)                                                   \
    do {                                                               \
        if (!(cond)) { fprintf(stderr, "line %d: %s\n", __LINE__, #cond); bad = 1; } \
    } while (0)

int main() {
    const int32_t fib[15] = {1, 2, 3, 5, 8, 13, 21, 34, 55, 89, 144, 233, 377, 610, 987};
    void *p = (void *)4096;
    float *f = (float *)4096;
    const fibattn_layout_t odd[8] = {{4096, 1024, 64}, {4096, 1024, 64}, {4096, 1024, 64}, {4096, 1024, 64},
                                     {4096, 1024, 64}, {4096, 1024, 64}, {4096, 1024, 64}, {4096, 1024, 3}};
    for (int T : {-1, 0, 1, 7, 1024, 1 << 24, 0x7fffffff})
        for (int H : {0, 1, 8, 65536, 0x7fffffff})
            for (int Hkv : {-3, 0, 1, 3, 8})
                for (int D : {0, 32, 64, 128, 130})
                    for (const void *table : {(const void *)nullptr, (const void *)p})
                        // never enough workspace: every size that is not refused itself ends there
                        EXPECT(fibattn_backward_joined(p, p, p, p, f, p, p, p, p, f, nullptr, p, 0, nullptr, 2, H, Hkv, T, D,
                                                       8, fib, 15, 1.f, table, 0.f, FIBATTN_BF16, nullptr) != FIBATTN_OK);
    EXPECT(fibattn_backward_joined(p, p, p, p, f, p, p, p, p, f, nullptr, p, 1u << 30, odd, 2, 4, 2, 8, 64, 8, fib, 15, 1.f,
                                   nullptr, 0.f, FIBATTN_BF16, nullptr) == FIBATTN_ERR_INVALID_ARG);
    EXPECT(fibattn_backward_joined(p, p, p, p, f, p, p, p, p, f, f, p, 1u << 30, nullptr, 2, 4, 2, 8, 64, 8, fib, 15, 1.f,
                                   nullptr, 0.f, FIBATTN_BF16, nullptr) == FIBATTN_ERR_INVALID_ARG);
    EXPECT(fibattn_backward_joined(p, p, p, p, f, p, p, p, p, f, nullptr, p, 1u << 30, nullptr, 2, 4, 2, 8, 64, 8, nullptr, 15,
                                   1.f, nullptr, 0.f, (fibattn_dtype_t)9, nullptr) == FIBATTN_ERR_INVALID_ARG);
    printf(bad ? "FAILED\n" : "OK\n");
    return bad;
}
