// Runs the host-only parts of include/symb_block.h (argument checks and the work plans behind the workspace figures) under -fsanitize=address,undefined: ragged, empty, enormous
// and invalid batches.  No GPU call is made.  Prints one line; exit status 0 = every call returned what it should.
#include <climits>
#include <cstdio>
#include <vector>

#include "../../include/symb_block.h"

static unsigned lcg = 4242u;
static unsigned rnd(unsigned n) {
    lcg = lcg * 1664525u + 1013904223u;
    return (lcg >> 8) % n;
}

int main() {
    int fails = 0;
    double sum = 0;
    alignas(16) static unsigned char fake[4096];         // stands for device memory: never dereferenced by host-only calls
    for (int trial = 0; trial < 300; ++trial) {
        const int S = (int)rnd(60);
        std::vector<int32_t> off(S + 1, 0), past(S);
        std::vector<symb_norm> norms(S);
        for (int i = 0; i < S; ++i) {
            const unsigned k = rnd(6);
            off[i + 1] = off[i] + (k == 0 ? 0 : k < 3 ? 1 : (int)rnd(900));
            past[i] = rnd(3) ? (int)rnd(20000) : 0;
            norms[i] = symb_norm{fake, nullptr, rnd(3) ? fake + 16 * rnd(4) : nullptr, nullptr};
        }
        symb_norm_batch nb{8 * (1 + (int)rnd(2048)), S, off.data(), norms.data(), (int32_t)rnd(2), 1e-5f, (float)rnd(2)};
        size_t bytes = 0;
        fails += symb_norm_workspace_bytes(&nb, &bytes) != SYMB_OK;
        sum += (double)bytes;
        const int H[] = {1, 2, 3, 8, 16, 32}, G[] = {1, 2, 4, 8, 48}, P[] = {32, 64, 128};
        const int h = H[rnd(6)], g = G[rnd(5)], pt = P[rnd(3)];
        symb_kv_batch kb{S, off.data(), past.data(), nullptr, 40000};
        symb_kv_cache c{nullptr, nullptr, nullptr, nullptr, 1 + (int)rnd(1000), h, rnd(2) ? 64 : 128, pt};
        fails += symb_kv_workspace_bytes(&kb, &c, h * g, rnd(2) ? 0 : (int)rnd(5000), &bytes) != SYMB_OK;
        sum += (double)bytes;
        fails += symb_kv_workspace_bytes(&kb, &c, h * g + (h > 1), 0, &bytes) != (h > 1 ? SYMB_ERR_INVALID_ARG : SYMB_OK);
        if (S) {
            const int32_t keep = off[S];
            off[S] = -1;
            fails += symb_norm_workspace_bytes(&nb, &bytes) != SYMB_ERR_BAD_SEGMENTS;
            fails += symb_kv_workspace_bytes(&kb, &c, h, 0, &bytes) != SYMB_ERR_BAD_SEGMENTS;
            off[S] = keep;
            past[S - 1] = INT_MAX;
            fails += symb_kv_workspace_bytes(&kb, &c, h, 0, &bytes) == (off[S] > off[S - 1] ? SYMB_OK : SYMB_ERR_UNSUPPORTED);
        }
    }
    // one context of two thousand million tokens, and the same behind a window
    int32_t off[2] = {0, 1}, past[1] = {INT_MAX - 2048};
    symb_kv_batch kb{1, off, past, nullptr, INT_MAX / 32 + 1};
    symb_kv_cache c{nullptr, nullptr, nullptr, nullptr, 1, 1, 128, 32};
    size_t bytes = 0;
    fails += symb_kv_workspace_bytes(&kb, &c, 1, 0, &bytes) != SYMB_OK || !bytes;
    fails += symb_kv_workspace_bytes(&kb, &c, 1, 4096, &bytes) != SYMB_OK;
    fails += symb_kv_workspace_bytes(&kb, &c, 1, INT_MAX, &bytes) != SYMB_OK;
    std::printf("fails=%d sum=%.0f\n", fails, sum);
    return fails != 0;
}
