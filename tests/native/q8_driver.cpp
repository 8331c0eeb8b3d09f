// Drives the entry points of the 8-bit path through valid and invalid arguments
// with stub launchers (fake, never dereferenced addresses): the status, and
// whether a launch was reached.  Built with sanitizers.
#include <cstdio>

#include "cpdp_q8.h"

extern int g_launches;
static int failures = 0;

#define EXPECT(call, want, launched)                                                   \
    do {                                                                               \
        const int before = g_launches, got = (call);                                   \
        if (got != (want) || (g_launches != before) != (launched)) {                   \
            std::printf("FAIL line %d: status %d (want %d), launched %d\n", __LINE__, got, \
                        (int)(want), (int)(g_launches != before));                     \
            ++failures;                                                                \
        }                                                                              \
    } while (0)

static void* at(int k) {
    return reinterpret_cast<void*>((uintptr_t)(1ull << 40) + ((uintptr_t)k << 36));
}
static int8_t* q(int k) { return static_cast<int8_t*>(at(k)); }
static float* f(int k) { return static_cast<float*>(at(k)); }

int main() {
    const int64_t T = 8, D = 60, L = 64, big = (int64_t)1 << 20;
    EXPECT(cpdp_q8_rows(at(0), L, 1, T, D, q(1), L, f(2), nullptr, 0, 9, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_rows(at(0), L, 1, T, D, q(1), L, f(2), at(3), L, 0, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_rows(at(0), L, 1, 0, D, nullptr, L, nullptr, nullptr, 0, 0, nullptr), CPDP_OK, false);
    EXPECT(cpdp_q8_rows(at(0), L, 1, T, D, q(0), L, f(2), nullptr, 0, 0, nullptr), CPDP_ERR_OVERLAP, false);
    EXPECT(cpdp_q8_rows(at(0), (int64_t)1 << 62, 1, T, D, q(1), L, f(2), nullptr, 0, 0, nullptr), CPDP_ERR_INVALID_ARG, false);
    EXPECT(cpdp_q8_rows(at(0), INT64_MIN, 1, T, D, q(1), L, f(2), nullptr, 0, 0, nullptr), CPDP_ERR_INVALID_ARG, false);
    EXPECT(cpdp_q8_rows(at(0), L, 1, INT64_MAX, D, q(1), L, f(2), nullptr, 0, 0, nullptr), CPDP_ERR_INVALID_ARG, false);
    EXPECT(cpdp_q8_values(q(0), L, f(1), T, D, at(2), L, 0, nullptr), CPDP_OK, true);
    // in place on the input and on the residual, and on rows of another stride
    EXPECT(cpdp_q8_norm(at(0), L, at(1), L, 0, at(2), 0, 0.0f, T, D, at(0), L, q(3), L, f(4), nullptr, nullptr, 0, 0, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_norm(at(0), L, at(1), L, 0, at(2), 0, 0.0f, T, D, at(1), L, q(3), L, f(4), f(5), at(6), L, 1, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_norm(at(0), L, at(1), L, 0, at(2), 0, 0.0f, T, D, at(1), 2 * L, q(3), L, f(4), nullptr, nullptr, 0, 0, nullptr), CPDP_ERR_OVERLAP, false);
    EXPECT(cpdp_q8_norm(at(0), L, nullptr, 0, 0, at(2), 1, 1e-6f, T, D, nullptr, 0, q(3), L, f(4), nullptr, nullptr, 0, 0, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_norm_bwd(at(0), L, at(1), L, nullptr, 0, 1, at(2), 0, f(3), T, D, at(4), L, at(5), 1, at(6), big, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_norm_bwd(at(0), L, at(1), L, nullptr, 0, 1, at(2), 0, f(3), 0, D, at(4), L, at(5), 1, at(6), big, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_norm_bwd(at(0), L, at(1), L, nullptr, 0, 1, at(2), 0, f(3), T, D, at(4), L, at(5), 1, at(6), 8, nullptr), CPDP_ERR_INVALID_ARG, false);
    EXPECT(cpdp_q8_matmul(q(0), L, f(1), q(2), L, f(3), T, 20, D, at(4), 24, 1, at(5), big, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_matmul(q(0), L, f(1), q(0), L, f(1), T, T, D, at(4), 24, 1, at(5), big, nullptr), CPDP_OK, true);  // a a^T
    EXPECT(cpdp_q8_matmul(q(0), L, f(1), q(2), L, f(3), T, 0, D, nullptr, 0, 1, nullptr, 0, nullptr), CPDP_OK, false);
    EXPECT(cpdp_q8_matmul(q(0), L, f(1), q(2), L, f(3), T, 20, 131072, at(4), 24, 1, at(5), big, nullptr), CPDP_ERR_INVALID_ARG, false);
    // g and u, dg and du as halves of one matrix; halves that overlap
    EXPECT(cpdp_q8_act(1, at(0), static_cast<char*>(at(0)) + 2 * L, 2 * L, 1, T, D, q(1), L, f(2), nullptr, 0, 0, nullptr, nullptr, nullptr, nullptr, 0, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_act(1, at(0), at(1), L, 1, T, D, q(2), L, f(3), nullptr, 0, 0, q(4), f(5), q(4) + L, f(6), 2 * L, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_act(1, at(0), at(1), L, 1, T, D, q(2), L, f(3), nullptr, 0, 0, q(4), f(5), nullptr, f(6), 2 * L, nullptr), CPDP_ERR_NULL, false);
    EXPECT(cpdp_q8_act(0, at(0), nullptr, L, 1, T, D, q(2), L, f(3), nullptr, 0, 0, q(4), f(5), nullptr, nullptr, L, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_act_bwd(1, at(0), L, 1, q(1), f(2), q(3), f(4), L, T, D, at(5), static_cast<char*>(at(5)) + 2 * L, 2 * L, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_act_bwd(1, at(0), L, 1, q(1), f(2), q(3), f(4), L, T, D, at(5), static_cast<char*>(at(5)) + L, 2 * L, nullptr), CPDP_ERR_OVERLAP, false);
    EXPECT(cpdp_q8_act_bwd(1, at(0), L, 1, q(1), f(2), q(3), f(4), L, T, D, static_cast<char*>(at(5)) + 2 * L, at(5), 2 * L, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_act_bwd(2, at(0), L, 1, q(1), f(2), q(3), f(4), L, T, D, at(5), at(6), L, nullptr), CPDP_ERR_INVALID_ARG, false);
    EXPECT(cpdp_q8_grad_input(at(0), L, 1, q(1), L, f(2), T, 20, D, at(3), L, 0, at(4), big, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_grad_input(nullptr, 0, 1, nullptr, 0, nullptr, T, 0, D, at(3), L, 0, nullptr, 0, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_grad_input(at(0), L, 1, q(1), L, f(2), 0, 20, D, at(3), L, 0, nullptr, 0, nullptr), CPDP_OK, false);
    EXPECT(cpdp_q8_grad_weight(at(0), L, 0, q(1), L, f(2), T, 20, D, at(3), L, 0, at(4), big, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_grad_weight(nullptr, 0, 0, nullptr, 0, nullptr, 0, 20, D, at(3), L, 0, nullptr, 0, nullptr), CPDP_OK, true);
    EXPECT(cpdp_q8_grad_weight(at(0), L, 0, q(1), L, f(2), T, 20, D, at(3), L, 0, at(4), 0, nullptr), CPDP_ERR_INVALID_ARG, false);
    if (failures == 0) std::printf("OK\n");
    return failures != 0;
}
