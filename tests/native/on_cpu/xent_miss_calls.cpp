// Makes the calls of the loss that hand on a token's miss on the CPU, as xent_calls does of
// the others: a line of stdin is a call and its sizes.
//   xent_miss      T V K
//   xent_miss_bwd  T V K dx_dt dw_dt (-1: left out)
#define main q8_calls_main
#include "q8_calls.cpp"
#undef main

namespace {

int call_loss(const std::string& op, const int64_t* v) {
    Memory m;
    const int64_t T = v[0], V = v[1], K = v[2];
    const bool whole = op != "xent_miss";  // (up to the end of a row's last 16 bytes)
    const Rows x = matrix(m, T, K, 1, whole), w = matrix(m, V, K, 1, whole), none{nullptr, 0};
    float* xs = m.vector(T);
    float* ws = m.vector(V);
    auto* target = reinterpret_cast<int64_t*>(m.take(T * 8));
    // the first and last class, one between, none, and one that is not there
    if (running)
        for (int64_t t = 0; t < T; ++t)
            target[t] = t % 5 == 0 ? 0 : t % 5 == 1 ? V - 1 : t % 5 == 2 ? t % V : t % 5 == 3 ? -1 : V;
    if (op == "xent_miss") {
        const int64_t bytes = cpdp_q8_xent_workspace(T, V, K);
        return cpdp_q8_xent_miss(x.q(), x.ld, xs, w.q(), w.ld, ws, target, T, V, K, m.vector(T),
                                 m.vector(T), m.vector(T), m.take(bytes), bytes, nullptr);
    }
    const int dx_dt = (int)(v[3] < 0 ? v[4] : v[3]), dw_dt = (int)(v[4] < 0 ? v[3] : v[4]);
    const int64_t bytes = cpdp_q8_xent_bwd_workspace(T, V, K, dx_dt, dw_dt);
    const Rows dx = v[3] < 0 ? none : matrix(m, T, K, size_of(dx_dt));
    const Rows dw = v[4] < 0 ? none : matrix(m, V, K, size_of(dw_dt));
    return cpdp_q8_xent_miss_bwd(x.q(), x.ld, xs, w.q(), w.ld, ws, target, m.vector(T),
                                 m.vector(T), m.vector(T), T, V, K, dx.p, dx.ld, dx_dt, dw.p,
                                 dw.ld, dw_dt, m.take(bytes), bytes, nullptr);
}

}  // namespace

int main(int argc, char** argv) {
    running = argc > 1 && std::string(argv[1]) == "run";
    char line[256];
    while (fgets(line, sizeof(line), stdin) != nullptr) {
        char op[32];
        long long w[8] = {};
        sscanf(line, "%31s %lld %lld %lld %lld %lld", op, w, w + 1, w + 2, w + 3, w + 4);
        int64_t v[8];
        for (int i = 0; i < 8; ++i) v[i] = w[i];
        if (running) fprintf(stderr, "%s", line), fflush(stderr);
        launched.clear();
        const int status = call_loss(op, v);
        printf("%d%s%s\n", status, launched.c_str(), too_large ? " too large" : "");
        fflush(stdout);
        too_large = false;
    }
    return 0;
}
