// Makes calls of gradient norms and clipping on the CPU, every thread of every launch, on
// buffers of exactly the bytes that they may touch (what lies between the rows is poisoned):
// a line of stdin is a call, the line that answers it its status.
//   flat  W P bf16 mean clip
//   plan  W mean clip numel...
#include <hip/hip_runtime.h>
#include <sanitizer/asan_interface.h>
#include <stdio.h>
#include <stdlib.h>

#include <sstream>
#include <string>
#include <vector>

#include "clip_launch.h"
#include "cpdp.h"
#include "plan_check.h"

dim3 threadIdx, blockIdx, blockDim, gridDim;
static bool too_large = false;
bool on_launch(const void*, dim3 grid, dim3 block) {
    too_large |= (uint64_t)grid.x * block.x >> 32 != 0;
    return true;
}

namespace cpdp {
constexpr int64_t kChunk = 256;
int64_t coords_per_block() { return kChunk; }
// (plans are made here)
int check_plan_handle(const cpdp_plan*) { return CPDP_OK; }
}  // namespace cpdp

namespace {

// Gradients that are long: 3.4e38 each
char* take(std::vector<char*>& held, size_t bytes) {
    void* p = nullptr;
    if (posix_memalign(&p, 16, bytes == 0 ? 1 : bytes) != 0) abort();
    memset(p, 0x7f, bytes);
    held.push_back(static_cast<char*>(p));
    return static_cast<char*>(p);
}

int flat(std::istream& in, std::vector<char*>& held) {
    int W, bf16, mean, clip;
    int64_t P;
    in >> W >> P >> bf16 >> mean >> clip;
    const int64_t es = bf16 ? 2 : 4, row = P * es, ld = (row + 15) / 16 * 16 + 32;
    char* g = take(held, P == 0 ? 0 : (W - 1) * ld + row);
    for (int i = 0; P > 0 && i + 1 < W; ++i) ASAN_POISON_MEMORY_REGION(g + i * ld + row, ld - row);
    const int64_t need = cpdp_grad_norm_workspace(W, P);
    auto* norm = reinterpret_cast<float*>(take(held, 4 * (mean ? 1 : W)));
    char* ws = take(held, need);
    const int s = clip ? cpdp_clip_grads(g, W, P, ld / es, bf16, 1e-30f, mean, norm, ws, need, nullptr)
                       : cpdp_grad_norm(g, W, P, ld / es, bf16, mean, norm, ws, need, nullptr);
    for (int i = 0; P > 0 && i + 1 < W; ++i)
        ASAN_UNPOISON_MEMORY_REGION(g + i * ld + row, ld - row);
    return s;
}

int plan(std::istream& in, std::vector<char*>& held) {
    int W, mean, clip;
    in >> W >> mean >> clip;
    std::vector<int64_t> numel;
    for (int64_t x; in >> x;) numel.push_back(x);
    const int64_t n = (int64_t)numel.size();
    // (the layout that cpdp_launch.h documents)
    std::vector<int64_t> table = {W, n, 0, 0};
    int64_t chunks = 0;
    for (int64_t x : numel) {
        table.push_back(chunks);
        chunks += (x + cpdp::kChunk - 1) / cpdp::kChunk;
    }
    table.push_back(chunks);
    table[2] = chunks;
    for (int64_t x : numel) table.push_back(x);
    for (int family = 0; family < 4; ++family)
        for (int64_t i = 0; i < W * n; ++i)
            table.push_back(family == 3 && numel[i % n] > 0
                                ? reinterpret_cast<int64_t>(take(held, numel[i % n] * 4))
                                : 0);
    for (int64_t i = 0; i < 2 * n; ++i) table.push_back(0);
    cpdp_plan p{};
    p.table = table.data();
    p.W = W;
    p.n_tensors = (int)n;
    p.total_chunks = chunks;
    const int64_t need = cpdp_grad_norm_plan_workspace(&p);
    auto* norm = reinterpret_cast<float*>(take(held, 4 * (mean ? 1 : W)));
    char* ws = take(held, need);
    return clip ? cpdp_clip_grads_plan(&p, 1e-30f, mean, norm, ws, need, nullptr)
                : cpdp_grad_norm_plan(&p, mean, norm, ws, need, nullptr);
}

}  // namespace

int main() {
    char line[8192];
    while (fgets(line, sizeof(line), stdin) != nullptr) {
        fprintf(stderr, "%s", line);
        std::istringstream in(line);
        std::string op;
        in >> op;
        std::vector<char*> held;
        const int s = op == "flat" ? flat(in, held) : plan(in, held);
        for (char* p : held) free(p);
        printf("%d%s\n", s, too_large ? " large" : "");
        fflush(stdout);
    }
    return 0;
}
