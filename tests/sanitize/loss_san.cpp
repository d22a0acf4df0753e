// Runs the host-only parts of include/symb_loss.h (argument checks and the plan behind the workspace figures) under -fsanitize=address,undefined: ragged, empty, enormous and invalid batches.
// No GPU call is made.  Prints one line; exit status 0 = every call returned what it should.
#include <algorithm>
#include <climits>
#include <cstdio>
#include <vector>

#include "../../include/symb_loss.h"

static unsigned lcg = 77u;
static unsigned rnd(unsigned n) {
    lcg = lcg * 1664525u + 1013904223u;
    return (lcg >> 8) % n;
}

int main() {
    int fails = 0;
    double sum = 0;
    size_t bytes = 0;
    for (int trial = 0; trial < 400; ++trial) {
        const int S = (int)rnd(40);
        std::vector<int32_t> off(S + 1, 0);
        std::vector<symb_loss> losses(S, symb_loss{1.f, 2.f});
        for (int i = 0; i < S; ++i) off[i + 1] = off[i] + (rnd(5) ? (int)rnd(rnd(2) ? 30 : 3000) : 0);
        symb_loss_batch b{8 * (1 + (int)rnd(1024)), 1 + (int)rnd(rnd(2) ? 300000 : 700), S, off.data(), losses.data(), (int32_t)rnd(2), (float)rnd(2) * 30.f};
        for (int gradient = 0; gradient < 2; ++gradient) {
            fails += symb_loss_workspace_bytes(&b, 0, gradient, &bytes) != SYMB_OK || (off[S] > 0) != (bytes > 0);
            sum += (double)bytes;
            fails += symb_loss_workspace_bytes(&b, 1 + (int)rnd(1024), gradient, &bytes) != SYMB_OK;
            sum += (double)bytes;
        }
        if (S) {
            losses[rnd(S)].temperature = 0.f;
            fails += symb_loss_workspace_bytes(&b, 3, 1, &bytes) != SYMB_ERR_INVALID_ARG;
            off[S] = -1;
            fails += symb_loss_workspace_bytes(&b, 0, 1, &bytes) != SYMB_ERR_BAD_SEGMENTS;
        }
    }
    // the most rows, the largest vocabulary, the widest rows, and all of what is allowed at once
    symb_loss one{1.f, 1.f};
    for (const int64_t width : {8, 4096, 32768})
        for (const int vocab : {1, 300, 1 << 22}) {
            int32_t off[2] = {0, (int32_t)std::min<int64_t>((((int64_t)1 << 31) - 1) / width, SYMB_LOSS_MAX_ROWS)};
            symb_loss_batch b{(int32_t)width, vocab, 1, off, &one, 0, 0.f};
            for (int gradient = 0; gradient < 2; ++gradient) {
                fails += symb_loss_workspace_bytes(&b, 0, gradient, &bytes) != SYMB_OK;
                // rows' own figures, and what a chunk of them holds
                fails += (double)bytes > (double)off[1] * 64 + 8.5 * (1 << 30);
                fails += symb_loss_workspace_bytes(&b, 1024, gradient, &bytes) != SYMB_OK;
            }
            ++off[1];
            fails += symb_loss_workspace_bytes(&b, 0, 1, &bytes) != SYMB_ERR_UNSUPPORTED;
            off[1] = INT_MAX;
            fails += symb_loss_workspace_bytes(&b, 0, 1, &bytes) != SYMB_ERR_UNSUPPORTED;
        }
    std::printf("fails=%d sum=%.0f\n", fails, sum);
    return fails != 0;
}
