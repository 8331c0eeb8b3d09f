// Softmax cross entropy of 8-bit rows over the classes of 8-bit weights, and its
// gradients, without the logits being kept.
//
// More than 64 tokens (fewer: q8_xent_few.hip): tiles of the product of rows and weights whose results are used
// where they are made (q8_xent_tile.h).  The loss takes one launch over all tiles and
// one that joins what they found of each token.  Its gradients make the logits again, a
// piece of the classes at a time, and leave the gradient of them laid out for two
// products on the bf16 matrix cores (q8_grad_gemm.h).
#include "q8_grad_layout.h"
#include "q8_xent_tile.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int64_t kFewTokens = 64;

// Joins the tiles' parts of each row's statistics: 16 rows a block, 16 threads a row.
__global__ __launch_bounds__(256) void xent_join_kernel(const Stats* part, const float* hit,
                                                        int64_t T, int64_t tiles, int64_t V,
                                                        const int64_t* target, float* loss,
                                                        float* lse) {
    __shared__ Stats words[16][17];
    const int row = threadIdx.x % 16, slice = threadIdx.x / 16;
    const int64_t t = (int64_t)blockIdx.x * 16 + row, from = t < T ? t : T - 1;
    Stats s = {-__builtin_inff(), 0.0f};
    int64_t j = slice;
    for (; j + 48 < tiles; j += 64) {
        Stats v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = part[(j + 16 * i) * T + from];
#pragma unroll
        for (int i = 0; i < 4; ++i) s = join(s, v[i]);
    }
    for (; j < tiles; j += 16) s = join(s, part[j * T + from]);
    words[slice][row] = s;
    __syncthreads();
    if (slice != 0 || t >= T) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s = join(s, words[i][row]);
    write_loss(s, hit[t], target[t], V, lse + t, loss + t);
}

// f(tile) with the tile's size as a compile-time number
template <class F>
int with_tile(int tile, F f) {
    if (tile == 256) return f(Int<256>());
    if (tile == 128) return f(Int<128>());
    return f(Int<64>());
}
// wavefronts across a tile, LDS buffers of its loop, threads
constexpr int across(int tile) { return tile == 256 ? 4 : 2; }
constexpr int buffers(int tile) { return tile == 64 ? 4 : 2; }
constexpr int threads(int tile) { return 128 * across(tile); }

Logits logits_of(const Loss& l, int64_t first, int64_t n) {
    Logits z{};
    z.o.a = reinterpret_cast<const char*>(l.x.q);
    z.o.b = reinterpret_cast<const char*>(l.w.q + first * l.w.ld);
    z.o.lda = l.x.ld;
    z.o.ldb = l.w.ld;
    z.o.M = l.T;
    z.o.N = n;
    z.o.row = (int)l.K;
    z.x_scale = l.x.scale;
    z.w_scale = l.w.scale + first;
    z.target = l.target;
    z.first = first;
    return z;
}

struct ForwardRoom : Room {
    int tile;
    int64_t tiles, part, hit;
};
ForwardRoom forward_room(int64_t T, int64_t V, int64_t K) {
    ForwardRoom r;
    r.tile = logit_tile(T, V, up(K, kStep), 3500, 0);
    r.tiles = up(V, r.tile);
    if (r.tiles > 1) {
        r.part = r.take(r.tiles * T * (int64_t)sizeof(Stats));
        r.hit = r.take(T * 4);
    }
    return r;
}

int forward(const Loss& l, float* loss, float* lse, void* ws, void* stream) {
    const ForwardRoom r = forward_room(l.T, l.V, l.K);
    const bool one = r.tiles == 1;
    const Found to{one ? nullptr : at<Stats>(ws, r.part), one ? nullptr : at<float>(ws, r.hit), lse,
                   loss};
    const int e = with_tile(r.tile, [&](auto tile) {
        const int64_t tm = up(l.T, tile);
        // (a launch holds fewer than 2^32 work items)
        const int64_t most = (((int64_t)1 << 32) / threads(tile) - 1) / tm;
        for (int64_t j = 0; j < r.tiles; j += most) {
            const int64_t tn = r.tiles - j < most ? r.tiles - j : most, v = j * tile;
            const Logits z = logits_of(l, v, l.V - v < tn * tile ? l.V - v : tn * tile);
            if (int s = launch(xent_stats_kernel<tile, across(tile), buffers(tile)>,
                               dim3((uint32_t)(tm * tn)), threads(tile), stream, z, to, tm, tn, j))
                return s;
        }
        return 0;
    });
    if (e || one) return e;
    return launch(xent_join_kernel, dim3((uint32_t)up(l.T, 16)), 256, stream, to.part, to.hit, l.T,
                  r.tiles, l.V, l.target, loss, lse);
}

// 8-bit operands [R x C] as out [C x pad] in bf16, zeros from R to pad: two of them in a
// launch, or one (the other has no blocks).
__global__ __launch_bounds__(256) void xent_turn_kernel(Source a, Source b) {
    __shared__ Tile<1, tile_cols<int8_t>()> tile;
    if (blockIdx.x < a.blocks) transpose<I8, 1>(a, blockIdx.x, tile);
    else transpose<I8, 1>(b, blockIdx.x - (uint32_t)a.blocks, tile);
}
Source source(const int8_t* q, int64_t ld, int64_t R, int64_t C, int64_t pad, uint16_t* out) {
    return {q, ld, nullptr, R, C, out, pad, pad / 64 * up(C, tile_cols<int8_t>())};
}
int turn(const Source& a, const Source& b, void* stream) {
    const int64_t blocks = a.blocks + b.blocks;
    if (blocks == 0) return 0;
    if (blocks * 256 >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
    return launch(xent_turn_kernel, dim3((uint32_t)blocks), 256, stream, a, b);
}

// Classes of a piece: 2^27 logits' gradients at most (268 MB a part), whole tiles.
int64_t piece_of(int64_t T, int64_t V) {
    const int64_t n = ((int64_t)1 << 27) / T / 1024 * 1024;
    return n < 1024 ? (V < 1024 ? V : 1024) : n < V ? n : V;
}

struct BackwardRoom : Room {
    int64_t piece, row_ld, class_ld;  // classes of a piece; row lengths of the slopes
    int px, pw;                       // parts
    int64_t by_row, by_class, x, w, sum, slices;
};

// The tile of a gradient's product, and the slices that its sum over R is cut into where
// there are fewer tiles than CUs.  A step of a tile takes what it takes in grad_shape;
// here the large tiles are cut, too: dx of 4096 x 1024 over 32768 classes has 64 tiles of
// 256 x 256, and in 4 slices takes 260 us, in 256 tiles of 128 x 128 335.
// Whether a product is small: tiles that find a CU each, and few steps.  What it takes is
// mostly its launch, and two of them are made in one (128 x 100 x 384 fp32: two of 4.7 us,
// BOTH together).
bool small(int64_t M, int64_t N, int64_t R, int parts) {
    return up(M, 64) * up(N, 64) <= kCus / 2 && up(R, kRound) * parts <= 24;
}
Shape product_shape(int64_t M, int64_t N, int64_t R, int parts) {
    const int64_t steps = up(R, kRound);
    if (small(M, N, R, parts)) return {64, 64, 1, 0};
    struct {
        int bm, bn, passes, alone, each, end;
    } const tiles[] = {{256, 256, parts, 1800, 1800, 2000},
                       {256, 128, parts, 1100, 1100, 1500},
                       {128, 128, 1, 310 + 290 * parts, 230 + 390 * parts, 800},
                       {64, 64, 1, 250 + 100 * parts, 105 + 115 * parts, 500}};
    Shape best = {0, 0, 1, -1};
    for (const auto& t : tiles) {
        if (t.bm + t.bn == 384 && parts > 1) continue;
        const int64_t n = up(M, t.bm) * up(N, t.bn), all = steps * t.passes;
        if (t.bm < 256 && n >= (int64_t)1 << 23) continue;
        for (int slices = 1; slices <= 64; slices *= 2) {
            if (slices > 1 && (n * slices > (t.bm == 64 ? 2048 : 512) || all < 4 * slices)) break;
            const int64_t turns = up(n * slices, kCus);
            const double step = turns == 1 ? t.alone : (double)turns * t.each;
            const double time = (double)up(all, slices) * step + turns * t.end +
                                (slices > 1 ? 4500.0 + slices * (double)M * (double)N / 500.0 : 0);
            if (best.ns < 0 || time < best.ns) best = {t.bm, t.bn, slices, time};
        }
    }
    return best;
}

BackwardRoom backward_room(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    BackwardRoom r;
    r.piece = piece_of(T, V);
    r.row_ld = up(r.piece, kRound) * kRound;
    r.class_ld = up(T, kRound) * kRound;
    r.px = dx_bf16 ? 1 : 3;
    r.pw = dw_bf16 ? 1 : 3;
    r.by_row = r.take(r.px * T * r.row_ld * 2);
    r.by_class = r.take(r.pw * r.piece * r.class_ld * 2);
    r.x = r.take(K * r.class_ld * 2);
    r.w = r.take(K * r.row_ld * 2);
    const bool pieces = r.piece < V;
    if (pieces) r.sum = r.take(T * slices_ld(K) * 4);
    int64_t most = 0;
    const int64_t last = V - (V - 1) / r.piece * r.piece;
    for (int i = 0; i < 2; ++i) {
        const int64_t n = i ? last : r.piece;
        const int64_t a = pieces ? T * slices_ld(K) * 4 * product_shape(T, K, n, r.px).slices
                                 : slices_bytes(T, K, product_shape(T, K, n, r.px));
        const int64_t b = slices_bytes(n, K, product_shape(n, K, T, r.pw));
        most = a > most ? a : most;
        most = b > most ? b : most;
    }
    r.slices = r.take(most);
    return r;
}

template <int P>
int launch_tiles_of(const GradOperands& o, const Target& t, const Shape& s, void* stream) {
    if (s.bn == 256) return launch_grad_tiles<256, 256, 2, 4, false, false, 1>(o, t, s.slices, stream);
    if constexpr (P == 1)
        if (s.bm == 256)
            return launch_grad_tiles<256, 128, 4, 2, false, false, 1>(o, t, s.slices, stream);
    if (s.bm == 128) return launch_grad_tiles<128, 128, 2, 2, false, false, P>(o, t, s.slices, stream);
    return launch_grad_tiles<64, 64, 2, 2, false, false, P>(o, t, s.slices, stream);
}

// c [M x N] = the product of A, laid out in parts, and B, laid out, over R values.
// Without c, the slices (one at least) are left for xent_add_kernel.
struct Product {
    GradOperands o;
    Target t;
    Shape shape;
    bool join;
};
Product product_of(const uint16_t* a, int64_t a_part, const uint16_t* b, int64_t ld, int64_t M,
                   int64_t N, int64_t R, int parts, Mat c, void* slices) {
    Product p{};
    p.o.a = reinterpret_cast<const char*>(a);
    p.o.lda = p.o.ldb = ld * 2;
    p.o.a_part = a_part * 2;
    p.o.b = reinterpret_cast<const char*>(b);
    p.o.R = R;
    p.o.M = M;
    p.o.N = N;
    p.o.steps = (int)up(R, kRound);
    p.o.parts = parts;
    p.t.c = c.p != nullptr ? c.p : slices;
    p.t.ldc = c.p != nullptr ? c.ld : slices_ld(N);
    p.t.bf16 = c.p != nullptr && c.bf16;
    p.t.ws = slices;
    p.t.ldws = slices_ld(N);
    p.t.slice = M * p.t.ldws;
    p.shape = product_shape(M, N, R, parts);
    p.join = c.p != nullptr && p.shape.slices > 1;
    return p;
}
int launch_product(const Product& p, void* stream) {
    if (int e = p.o.parts == 1 ? launch_tiles_of<1>(p.o, p.t, p.shape, stream)
                               : launch_tiles_of<3>(p.o, p.t, p.shape, stream))
        return e;
    return p.join ? launch_join<Bf16>(p.t, p.o.M, p.o.N, p.shape.slices, stream) : 0;
}

// Two small products in one launch, blockIdx.y the one.
template <int P>
__global__ __launch_bounds__(256) void xent_both_kernel(GradOperands a, Target to_a,
                                                        GradOperands b, Target to_b) {
    const bool second = blockIdx.y != 0;
    const GradOperands o = second ? b : a;
    const int64_t tm = (o.M + 63) / 64, tn = (o.N + 63) / 64;
    if (blockIdx.x >= tm * tn) return;
    GradGemm<64, 64, 2, 2, false, false, P, 4>::run(o, second ? to_b : to_a, tm, tn, 1);
}
// Whether they may be: of as many parts, and small.
bool both_small(const Product& a, const Product& b) {
    return a.o.parts == b.o.parts && small(a.o.M, a.o.N, a.o.R, a.o.parts) &&
           small(b.o.M, b.o.N, b.o.R, b.o.parts);
}
int launch_both(const Product& a, const Product& b, void* stream) {
    const int64_t na = up(a.o.M, 64) * up(a.o.N, 64), nb = up(b.o.M, 64) * up(b.o.N, 64);
    const dim3 grid((uint32_t)(na > nb ? na : nb), 2);
    return a.o.parts == 3
               ? launch(xent_both_kernel<3>, grid, 256, stream, a.o, a.t, b.o, b.t)
               : launch(xent_both_kernel<1>, grid, 256, stream, a.o, a.t, b.o, b.t);
}

// sum <- sum and the slices of a piece, to dx after the last piece; 4 columns a thread
__global__ __launch_bounds__(256) void xent_add_kernel(float* sum, const float* part, int64_t ld,
                                                       int64_t slice, int64_t T, int64_t K,
                                                       int slices, int first, int last,
                                                       Target out) {
    const int64_t across = (K + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t t = i / across, k = i % across * 4;
    if (t >= T) return;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!first) x = *reinterpret_cast<const f32x4*>(sum + t * ld + k);
    for (int z = 0; z < slices; ++z)
        x += *reinterpret_cast<const f32x4*>(part + z * slice + t * ld + k);
    if (!last) {
        *reinterpret_cast<f32x4*>(sum + t * ld + k) = x;
        return;
    }
    const float v[4] = {x[0], x[1], x[2], x[3]};
    store_cols<4>(out, t, k, (int)(K - k < 4 ? K - k : 4), v);
}
int add(const BackwardRoom& r, void* ws, const Loss& l, int slices, bool first, bool last, Mat dx,
        void* stream) {
    Target out{};
    out.c = dx.p;
    out.ldc = dx.ld;
    out.bf16 = dx.bf16;
    const int64_t ld = slices_ld(l.K), across = up(l.K, 4);
    // (a launch holds fewer than 2^32 work items)
    return in_parts(l.T, across, [&](int64_t t, int64_t n) {
        Target part = out;
        part.c = static_cast<char*>(out.c) + t * out.ldc * (out.bf16 ? 2 : 4);
        return launch(xent_add_kernel, dim3((uint32_t)up(n * across, 256)), 256, stream,
                      at<float>(ws, r.sum) + t * ld, at<const float>(ws, r.slices) + t * ld, ld,
                      l.T * ld, n, l.K, slices, (int)first, (int)last, part);
    });
}

template <int PX, int PW>
int launch_slopes(const Logits& z, const Slopes& to, int64_t K, void* stream) {
    return with_tile(logit_tile(z.o.M, z.o.N, up(K, kStep), 0, PX + PW), [&](auto tile) {
        const int64_t tm = up(z.o.M, tile), tn = up(z.o.N, tile);
        if (tm * tn * threads(tile) >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
        return launch(xent_slopes_kernel<tile, across(tile), buffers(tile), PX, PW>,
                      dim3((uint32_t)(tm * tn)), threads(tile), stream, z, to, tm, tn);
    });
}

int backward(const Loss& l, const float* lse, const float* g, Mat dx, Mat dw, void* ws,
             void* stream) {
    const BackwardRoom r = backward_room(l.T, l.V, l.K, dx.bf16, dw.bf16);
    const bool x = dx.p != nullptr, w = dw.p != nullptr;
    for (int64_t v = 0; v < l.V; v += r.piece) {
        const int64_t n = l.V - v < r.piece ? l.V - v : r.piece;
        const Logits z = logits_of(l, v, n);
        Slopes to{};
        to.by_row = at<uint16_t>(ws, r.by_row);
        to.by_class = at<uint16_t>(ws, r.by_class);
        to.row_ld = up(n, kRound) * kRound;
        to.row_part = l.T * to.row_ld;
        to.class_ld = r.class_ld;
        to.class_part = n * r.class_ld;
        to.lse = lse;
        to.g = g;
        to.classes = l.V;
        const int px = x ? r.px : 0, pw = w ? r.pw : 0;
        const int e = px == 0   ? pw == 1 ? launch_slopes<0, 1>(z, to, l.K, stream)
                                          : launch_slopes<0, 3>(z, to, l.K, stream)
                      : px == 1 ? pw == 0   ? launch_slopes<1, 0>(z, to, l.K, stream)
                                  : pw == 1 ? launch_slopes<1, 1>(z, to, l.K, stream)
                                            : launch_slopes<1, 3>(z, to, l.K, stream)
                      : pw == 0 ? launch_slopes<3, 0>(z, to, l.K, stream)
                      : pw == 1 ? launch_slopes<3, 1>(z, to, l.K, stream)
                                : launch_slopes<3, 3>(z, to, l.K, stream);
        if (e) return e;
        auto* turned_x = at<uint16_t>(ws, r.x);
        auto* turned_w = at<uint16_t>(ws, r.w);
        const Source none{};
        if (int s = turn(w && v == 0 ? source(l.x.q, l.x.ld, l.T, l.K, r.class_ld, turned_x) : none,
                         x ? source(l.w.q + v * l.w.ld, l.w.ld, n, l.K, to.row_ld, turned_w) : none,
                         stream))
            return s;
        void* slices = at<char>(ws, r.slices);
        const bool whole = r.piece == l.V;
        Product of_x{}, of_w{};
        if (x)
            of_x = product_of(to.by_row, to.row_part, turned_w, to.row_ld, l.T, l.K, n, px,
                             whole ? dx : Mat{nullptr, 0, false}, slices);
        if (w)
            of_w = product_of(to.by_class, to.class_part, turned_x, r.class_ld, n, l.K, l.T, pw,
                             Mat{static_cast<char*>(dw.p) + v * dw.ld * (dw.bf16 ? 2 : 4), dw.ld,
                                 dw.bf16},
                             slices);
        if (x && w && whole && both_small(of_x, of_w)) return launch_both(of_x, of_w, stream);
        if (x) {
            if (int s = launch_product(of_x, stream)) return s;
            if (!whole)
                if (int s = add(r, ws, l, of_x.shape.slices, v == 0, v + n == l.V, dx, stream))
                    return s;
        }
        if (w)
            if (int s = launch_product(of_w, stream)) return s;
    }
    return 0;
}

}  // namespace

int64_t xent_workspace(int64_t T, int64_t V, int64_t K) {
    return T <= kFewTokens ? few_xent_workspace(T, V, K) : forward_room(T, V, K).bytes;
}

int launch_xent(const Loss& l, float* loss, float* lse, void* workspace, void* stream) {
    return l.T <= kFewTokens ? launch_few_xent(l, loss, lse, workspace, stream)
                             : forward(l, loss, lse, workspace, stream);
}

int64_t xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    return T <= kFewTokens ? few_xent_bwd_workspace(T, V, K, dx_bf16, dw_bf16)
                           : backward_room(T, V, K, dx_bf16, dw_bf16).bytes;
}

int launch_xent_bwd(const Loss& l, const float* lse, const float* g, Mat dx, Mat dw,
                    void* workspace, void* stream) {
    // a sum over no tokens
    if (l.T == 0)
        return launch_grad_weight(Mat{nullptr, 0, false}, l.x, 0, l.V, l.K, dw, workspace, stream);
    return l.T <= kFewTokens ? launch_few_xent_bwd(l, lse, g, dx, dw, workspace, stream)
                             : backward(l, lse, g, dx, dw, workspace, stream);
}

}  // namespace q8
}  // namespace cpdp
