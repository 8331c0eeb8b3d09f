// Makes calls of the 8-bit path's C ABI on the CPU (hip/hip_runtime.h here): a line of
// stdin is a call and its sizes, the line that answers it holds the kernels it launched.
//   q8_calls run    the kernels run, on buffers of exactly the bytes the header lets them
//                   read and write; what lies between the rows is poisoned
//   q8_calls note   they do not (addresses are made up)
#include <hip/hip_runtime.h>
#include <sanitizer/asan_interface.h>
#include <stdio.h>
#include <stdlib.h>

#include <memory>
#include <string>
#include <vector>

#include "cpdp_q8.h"

dim3 threadIdx, blockIdx, blockDim, gridDim;

namespace {

bool running = false;
std::string launched;
bool too_large = false;

// A buffer of `bytes`, or in note mode an address that nothing reads.
class Memory {
  public:
    ~Memory() {
        for (auto& b : held_) {
            ASAN_UNPOISON_MEMORY_REGION(b.first, b.second);
            free(b.first);
        }
    }
    char* take(size_t bytes) {
        if (!running) return reinterpret_cast<char*>(next_ += (uintptr_t)1 << 44);
        // (AddressSanitizer keeps 16 bytes or more around it)
        void* p = nullptr;
        if (posix_memalign(&p, 16, bytes == 0 ? 1 : bytes) != 0) abort();
        memset(p, 1, bytes);
        held_.emplace_back(p, bytes);
        return static_cast<char*>(p);
    }
    float* vector(int64_t n, int64_t element = 4) {
        return reinterpret_cast<float*>(take(n * element));
    }

  private:
    std::vector<std::pair<void*, size_t>> held_;
    uintptr_t next_ = 0;
};

struct Rows {
    char* p;
    int64_t ld;  // elements
    operator const void*() const { return p; }
    int8_t* q() const { return reinterpret_cast<int8_t*>(p); }
};
// rows x cols elements of `es` bytes, 32 bytes or more from row to row's end; with `whole`
// a row may be read up to the end of its last 16 bytes
Rows matrix(Memory& m, int64_t rows, int64_t cols, int64_t es, bool whole = false) {
    const int64_t row = cols * es, there = whole ? (row + 15) / 16 * 16 : row;
    const int64_t ld = (row + 15) / 16 * 16 + 32;
    const int64_t bytes = rows == 0 ? 0 : (rows - 1) * ld + there;
    Rows r{m.take(bytes), ld / es};
    if (running)
        for (int64_t i = 0; i + 1 < rows; ++i)
            ASAN_POISON_MEMORY_REGION(r.p + i * ld + there, ld - there);
    return r;
}

int64_t size_of(int dt) { return dt == CPDP_BF16 ? 2 : 4; }

int call(const std::string& op, const int64_t* v) {
    Memory m;
    const auto out = [&](int64_t r, int64_t c, int dt) { return matrix(m, r, c, size_of(dt)); };
    if (op == "rows") {  // T D x_dt y_dt (-1: no y)
        const int64_t T = v[0], D = v[1];
        const Rows x = out(T, D, v[2]), q = matrix(m, T, D, 1);
        const Rows y = v[3] < 0 ? Rows{nullptr, 0} : out(T, D, v[3]);
        return cpdp_q8_rows(x, x.ld, v[2], T, D, q.q(), q.ld, m.vector(T), y.p, y.ld, v[3],
                            nullptr);
    }
    if (op == "values") {  // T D y_dt
        const int64_t T = v[0], D = v[1];
        const Rows q = matrix(m, T, D, 1), y = out(T, D, v[2]);
        return cpdp_q8_values(q.q(), q.ld, m.vector(T), T, D, y.p, y.ld, v[2], nullptr);
    }
    if (op == "norm") {  // T D act_dt w_dt residual y_dt
        const int64_t T = v[0], D = v[1];
        const Rows x = out(T, D, v[2]), q = matrix(m, T, D, 1), none{nullptr, 0};
        const Rows r = v[4] ? out(T, D, v[2]) : none, h = v[4] ? out(T, D, v[2]) : none;
        const Rows y = v[5] < 0 ? none : out(T, D, v[5]);
        return cpdp_q8_norm(x, x.ld, r.p, r.ld, v[2], m.vector(D, size_of(v[3])), v[3], 1e-6f, T,
                            D, h.p, h.ld, q.q(), q.ld, m.vector(T), m.vector(T), y.p, y.ld, v[5],
                            nullptr);
    }
    if (op == "norm_bwd") {  // T D act_dt w_dt dres dw_dt
        const int64_t T = v[0], D = v[1], bytes = cpdp_q8_norm_bwd_workspace(T, D);
        const Rows dy = out(T, D, v[2]), h = out(T, D, v[2]), dx = out(T, D, v[2]);
        const Rows r = v[4] ? out(T, D, v[2]) : Rows{nullptr, 0};
        return cpdp_q8_norm_bwd(dy, dy.ld, h, h.ld, r.p, r.ld, v[2], m.vector(D, size_of(v[3])),
                                v[3], m.vector(T), T, D, dx.p, dx.ld, m.vector(D, size_of(v[5])),
                                v[5], m.take(bytes), bytes, nullptr);
    }
    if (op == "product") {  // M N K y_dt
        const int64_t M = v[0], N = v[1], K = v[2], bytes = cpdp_q8_matmul_workspace(M, N, K);
        const Rows a = matrix(m, M, K, 1), b = matrix(m, N, K, 1), y = out(M, N, v[3]);
        return cpdp_q8_matmul(a.q(), a.ld, m.vector(M), b.q(), b.ld, m.vector(N), M, N, K, y.p,
                              y.ld, v[3], m.take(bytes), bytes, nullptr);
    }
    if (op == "act") {  // kind T F act_dt y_dt checkpoint
        const int64_t T = v[1], F = v[2];
        const Rows g = out(T, F, v[3]), u = out(T, F, v[3]), q = matrix(m, T, F, 1);
        const Rows none{nullptr, 0}, y = v[4] < 0 ? none : out(T, F, v[4]);
        const Rows cg = v[5] ? matrix(m, T, F, 1) : none, cu = v[5] ? matrix(m, T, F, 1) : none;
        return cpdp_q8_act(v[0], g, u, g.ld, v[3], T, F, q.q(), q.ld, m.vector(T), y.p, y.ld, v[4],
                           cg.q(), v[5] ? m.vector(T) : nullptr, v[0] ? cu.q() : nullptr,
                           v[5] && v[0] ? m.vector(T) : nullptr, cg.ld, nullptr);
    }
    if (op == "act_bwd") {  // kind T F act_dt
        const int64_t T = v[1], F = v[2];
        const Rows da = out(T, F, v[3]), dg = out(T, F, v[3]), du = out(T, F, v[3]);
        const Rows cg = matrix(m, T, F, 1), cu = matrix(m, T, F, 1);
        return cpdp_q8_act_bwd(v[0], da, da.ld, v[3], cg.q(), m.vector(T), cu.q(), m.vector(T),
                               cg.ld, T, F, dg.p, du.p, dg.ld, nullptr);
    }
    // T N K dy_dt out_dt
    const int64_t T = v[0], N = v[1], K = v[2];
    const bool input = op == "grad_input";
    if (!input && op != "grad_weight") return -1;
    const int64_t R = input ? N : T;  // rows of the 8-bit operand
    const int64_t bytes =
        (input ? cpdp_q8_grad_input_workspace : cpdp_q8_grad_weight_workspace)(T, N, K, v[3], v[4]);
    const Rows dy = matrix(m, T, N, size_of(v[3]), true), q = matrix(m, R, K, 1, true);
    const Rows c = out(input ? T : N, K, v[4]);
    return (input ? cpdp_q8_grad_input : cpdp_q8_grad_weight)(
        dy, dy.ld, v[3], q.q(), q.ld, m.vector(R), T, N, K, c.p, c.ld, v[4], m.take(bytes), bytes,
        nullptr);
}

}  // namespace

bool on_launch(const void* kernel, dim3 grid, dim3 block) {
    char text[32];
    snprintf(text, sizeof(text), " %zx", reinterpret_cast<size_t>(kernel));
    launched += text;
    // (a launch holds fewer than 2^32 work items in a direction)
    too_large |= (uint64_t)grid.x * block.x >> 32 != 0 || grid.y > 65535;
    return running;
}

int main(int argc, char** argv) {
    running = argc > 1 && std::string(argv[1]) == "run";
    char line[256];
    while (fgets(line, sizeof(line), stdin) != nullptr) {
        char op[32];
        long long w[8] = {};
        sscanf(line, "%31s %lld %lld %lld %lld %lld %lld", op, w, w + 1, w + 2, w + 3, w + 4, w + 5);
        int64_t v[8];
        for (int i = 0; i < 8; ++i) v[i] = w[i];
        if (running) fprintf(stderr, "%s", line), fflush(stderr);
        launched.clear();
        const int status = call(op, v);
        printf("%d%s%s\n", status, launched.c_str(), too_large ? " too large" : "");
        fflush(stdout);
        too_large = false;
    }
    return 0;
}
