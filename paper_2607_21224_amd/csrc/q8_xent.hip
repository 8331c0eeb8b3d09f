// Softmax cross entropy of 8-bit rows over the classes of 8-bit weights, and its
// gradients, without the logits being kept.
//
// Logits are made in tiles of the product of rows and weights, whose results are used where
// they are made (q8_xent_tile.h); very few tokens' otherwise (q8_xent_few.hip), as are the
// gradients' products of up to 64.  The loss takes one launch
// over all tiles, or two, and one that joins what they found of each token.  Its gradients
// make the logits again, a piece of the classes at a time, and leave the gradient of them
// laid out for two products of fp16 numbers.
#include "q8_xent_tile.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int64_t kFewTokens = 64;

// Joins the tiles' parts of each row's statistics: 16 rows a block, 16 threads a row.
__global__ __launch_bounds__(256) void xent_join_kernel(const Stats* part, const float* hit,
                                                        int64_t T, int64_t tiles, int64_t V,
                                                        const int64_t* target, LossOut to) {
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
    write_loss(s, hit[t], target[t], V, to, t);
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
    TwoTiles split;
    int64_t tiles, part, hit;
};
ForwardRoom forward_room(int64_t T, int64_t V, int64_t K) {
    ForwardRoom r;
    r.split = logit_tiles(T, V, up(K, kStep), 3500, 0);
    r.tiles = r.split.first / 256 + up(V - r.split.first, r.split.tile);
    if (r.tiles > 1) {
        r.part = r.take(r.tiles * T * (int64_t)sizeof(Stats));
        r.hit = r.take(T * 4);
    }
    return r;
}

// Statistics of classes v to v + n, the parts of whose tiles are `at` on
int launch_stats(const Loss& l, const Found& to, int tile, int64_t at, int64_t v, int64_t n,
                 void* stream) {
    return with_tile(tile, [&](auto tile) {
        const int64_t tm = up(l.T, tile);
        // (a launch holds fewer than 2^32 work items)
        const int64_t most = (((int64_t)1 << 32) / threads(tile) - 1) / tm;
        for (int64_t j = 0; j < n; j += most * tile) {
            const int64_t left = n - j < most * tile ? n - j : most * tile, tn = up(left, tile);
            if (int e = launch(xent_stats_kernel<tile, across(tile), buffers(tile)>,
                               dim3((uint32_t)(tm * tn)), threads(tile), stream,
                               logits_of(l, v + j, left), to, tm, tn, at + j / tile))
                return e;
        }
        return 0;
    });
}

int forward(const Loss& l, const LossOut& out, void* ws, void* stream) {
    const ForwardRoom r = forward_room(l.T, l.V, l.K);
    const bool one = r.tiles == 1;
    const Found to{one ? nullptr : at<Stats>(ws, r.part), one ? nullptr : at<float>(ws, r.hit),
                   out};
    const int64_t first = r.split.first;
    if (first > 0)
        if (int e = launch_stats(l, to, 256, 0, 0, first, stream)) return e;
    const int e = launch_stats(l, to, r.split.tile, first / 256, first, l.V - first, stream);
    if (e || one) return e;
    return launch(xent_join_kernel, dim3((uint32_t)up(l.T, 16)), 256, stream, to.part, to.hit, l.T,
                  r.tiles, l.V, l.target, out);
}

// ---- what the products of the gradients need first ----------------------------------

constexpr int kRound = kStep / 2;  // fp16 numbers in a step: rows are padded to whole steps

// An 8-bit operand [R x C] laid out as fp16 [C][copies][pad], zeros from R to pad: as many
// copies as the other operand has parts, the second over kSecond.
struct Source {
    const int8_t* q;
    int64_t ld, R, C;
    uint16_t* out;
    int64_t pad;
    int copies;
    int64_t blocks;  // of 64 rows and 128 columns
};
Source source(const int8_t* q, int64_t ld, int64_t R, int64_t C, uint16_t* out, int64_t pad,
              int copies) {
    return {q, ld, R, C, out, pad, copies, pad / 64 * up(C, 128)};
}

// (columns of 32 pairs of rows, a word more, so that the 64 lanes of a wavefront, 8 pairs of
// rows and 8 columns 8 apart, write to 64 banks)
using Turned = uint32_t[128][33];

__device__ __forceinline__ void turn(const Source& s, uint32_t block, Turned& tile) {
    const uint32_t down = (uint32_t)(s.pad / 64);
    const int64_t r0 = (int64_t)(block % down) * 64, c0 = (int64_t)(block / down) * 128;
    const int pair = (int)threadIdx.x / 8, col = (int)threadIdx.x % 8 * kPiece;
    Raw<I8> x[2][2] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t r = r0 + 2 * pair + i, c = c0 + h * 64 + col;
            const int n = s.C - c > kPiece ? kPiece : (int)(s.C - c);
            if (r < s.R && n > 0) x[h][i].load(s.q + r * s.ld + c, n, (int)(c < 8 ? c : 8));
        }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < kPiece; ++k)
            tile[h * 64 + col + k][pair] = halves(x[h][0][k], x[h][1][k]);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 128; h += 32) {
        const int c = h + (int)threadIdx.x / 8, w = (int)threadIdx.x % 8 * 4;
        if (c0 + c >= s.C) continue;
        u32x4 v = {tile[c][w], tile[c][w + 1], tile[c][w + 2], tile[c][w + 3]};
        uint16_t* out = s.out + (c0 + c) * s.copies * s.pad + r0 + 2 * w;
        *reinterpret_cast<u32x4*>(out) = v;
        if (s.copies == 1) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t word = v[k];
            const f16x2 two = __builtin_bit_cast(f16x2, word);
            v[k] = halves((float)two[0] / kSecond, (float)two[1] / kSecond);
        }
        *reinterpret_cast<u32x4*>(out + s.pad) = v;
    }
}

// What the slopes' scales are found from (see Slopes), in `blocks` parts, and ones.  (By one
// block, gradients of 65 x 131072 x 64 bf16 took 87 us, and take 70.)
struct Largest {
    Held x, w;
    const int64_t* target;
    const float* g;
    int64_t T, V, K;
    float* out;   // [2][kLargest]; 0 past the parts
    float* ones;  // [K]
    int blocks;   // 0: not wanted
};
constexpr int64_t kClasses = 4096, kTokens = 1024;  // of a part at a time
__device__ __forceinline__ float over_block(float x, float* words) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = x;
    __syncthreads();
    return fmaxf(fmaxf(words[0], words[1]), fmaxf(words[2], words[3]));
}
// |x|, 0 if it is not finite
__device__ __forceinline__ float size_of(float x) {
    return magnitude(x) < 0x7f800000u ? fabsf(x) : 0.0f;
}
__device__ __forceinline__ void find_largest(const Largest& s, int block, float (&words)[2][4]) {
    float w = 0.0f, x = 0.0f;
    for (int64_t first = block * kClasses; first < s.V; first += s.blocks * kClasses) {
        float some[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t v = first + i * 256 + threadIdx.x;
            some[i] = s.w.scale[v < s.V ? v : s.V - 1];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) w = fmaxf(w, size_of(some[i]));
    }
    for (int64_t first = block * kTokens; first < s.T; first += s.blocks * kTokens) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t t = first + i * 256 + threadIdx.x, at = t < s.T ? t : s.T - 1;
            const float f = size_of(s.g[at] * s.x.scale[at]);
            x = fmaxf(x, s.target[at] < 0 ? 0.0f : f);
        }
    }
    w = over_block(w, words[0]);
    x = over_block(x, words[1]);
    if (threadIdx.x == 0) {
        s.out[block] = w;
        s.out[kLargest + block] = x;
    }
    if (block == 0 && (int)threadIdx.x >= s.blocks && threadIdx.x < kLargest)
        s.out[threadIdx.x] = s.out[kLargest + threadIdx.x] = 0.0f;
    for (int64_t k = block * 256 + threadIdx.x; k < s.K; k += s.blocks * 256) s.ones[k] = 1.0f;
}

// Two operands, or one (the other has no blocks), and the largest scales.
__global__ __launch_bounds__(256) void xent_turn_kernel(Source a, Source b, Largest s) {
    __shared__ Turned tile;
    __shared__ float words[2][4];
    const uint32_t block = blockIdx.x - (uint32_t)s.blocks;
    if (blockIdx.x < (uint32_t)s.blocks) find_largest(s, (int)blockIdx.x, words);
    else if (block < a.blocks) turn(a, block, tile);
    else turn(b, block - (uint32_t)a.blocks, tile);
}
int launch_turn(const Source& a, const Source& b, const Largest& s, void* stream) {
    const int64_t blocks = a.blocks + b.blocks + s.blocks;
    if (blocks == 0) return 0;
    if (blocks * 256 >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
    return launch(xent_turn_kernel, dim3((uint32_t)blocks), 256, stream, a, b, s);
}

// ---- the products --------------------------------------------------------------------

// Classes of a piece: 2^27 slopes (268 MB a part) at most, whole tiles, one at least, and rows
// that a tile can address.
int64_t piece_of(int64_t T, int64_t V) {
    int64_t n = ((int64_t)1 << 27) / T / 256 * 256;
    n = n < 256 ? 256 : n > (int64_t)1 << 20 ? (int64_t)1 << 20 : n;
    return piece_size(V, up(V, n), 256);
}
// With dx, 512 MB of weights, laid out, at most, too.  A piece costs 50 to 100 us, its launches'
// ends (gradients of 128 x 151936 x 4096 bf16 1305 us in one piece with 1.3 GB of workspace, 1445
// in three with 0.46; fp32 2170 with 2.7 and 2540 with 0.55; with 512 MB for slopes and weights
// together, 8192 x 32768 x 4096 bf16 took 4800 us, and takes 4570).
int64_t piece_of(int64_t T, int64_t V, int64_t K, int px) {
    const int64_t slopes = piece_of(T, V), weights = ((int64_t)1 << 28) / (px * K) / 256 * 256;
    return slopes <= weights ? slopes : piece_size(V, up(V, weights < 256 ? 256 : weights), 256);
}

// Whether a product is small: tiles that find a CU each, and few steps.  What it takes is
// mostly its launch, and two of them are made in one (128 x 100 x 384: gradients in 13 us,
// and 18 with two).
bool small(int64_t M, int64_t N, int64_t steps) {
    return up(M, 64) * up(N, 64) <= kCus / 2 && steps <= 16;
}
// The tile of a gradient's product, and the slices that its sum is cut into where there are
// fewer tiles than CUs.  A step of a tile takes what it takes in shape_of; here the large
// tiles are cut, too: dx of 4096 x 1024 over 32768 classes has 64 tiles of 256 x 256, and is
// made in 4 slices (with dw an eighth less time than in tiles of 128 x 128 and 256 x 128,
// 750 and 844 us in bf16).
Shape product_shape(int64_t M, int64_t N, int64_t steps) {
    if (small(M, N, steps)) return {64, 64, 1, 0};
    struct {
        int bm, bn, alone, each, end;
    } const tiles[] = {{256, 256, 1800, 1800, 2000},
                       {256, 128, 1100, 1100, 1500},
                       {128, 128, 540, 620, 800},
                       {64, 64, 280, 220, 500}};
    Shape best = {0, 0, 1, -1};
    for (const auto& t : tiles) {
        const int64_t n = up(M, t.bm) * up(N, t.bn);
        if (t.bm < 256 && n >= (int64_t)1 << 23) continue;
        for (int slices = 1; slices <= 64; slices *= 2) {
            if (slices > 1 && (n * slices > (t.bm == 64 ? 2048 : 512) || steps < 4 * slices)) break;
            const int64_t turns = up(n * slices, kCus);
            const double step = turns == 1 ? t.alone : (double)turns * t.each;
            const double time = (double)up(steps, slices) * step + turns * t.end +
                                (slices > 1 ? 4500.0 + slices * (double)M * (double)N / 500.0 : 0);
            if (best.ns < 0 || time < best.ns) best = {t.bm, t.bn, slices, time};
        }
    }
    return best;
}

// c [M x N] = the product of A [M x length] and B [N x length], with rows scaled.
// Without c, the slices (one at least) are left for xent_add_kernel, not scaled.
struct Product {
    Operands o;
    Target t;
    Shape shape;
    bool join;
};
int64_t steps_of(int64_t length) { return length / kRound; }
Product product_of(const uint16_t* a, const uint16_t* b, int64_t length, int64_t M, int64_t N,
                   const float* rows, const float* ones, Mat c, void* slices) {
    Product p{};
    p.o.a = reinterpret_cast<const char*>(a);
    p.o.b = reinterpret_cast<const char*>(b);
    p.o.lda = p.o.ldb = length * 2;
    p.o.M = M;
    p.o.N = N;
    p.o.row = (int)(length * 2);
    const bool whole = c.p != nullptr;
    p.t.c = whole ? c.p : slices;
    p.t.ldc = whole ? c.ld : slices_ld(N);
    p.t.bf16 = whole && c.bf16;
    p.t.row_scale = whole ? rows : nullptr;
    p.t.col_scale = whole ? ones : nullptr;
    p.t.ws = slices;
    p.t.ldws = slices_ld(N);
    p.t.slice = M * p.t.ldws;
    p.shape = product_shape(M, N, steps_of(length));
    p.join = whole && p.shape.slices > 1;
    return p;
}
int launch_product(const Product& p, void* stream) {
    const Shape& s = p.shape;
    const int e = s.bn == 256 ? launch_tiles<Half, 256, 256, 2, 4>(p.o, p.t, s.slices, stream)
                  : s.bm == 256
                      ? launch_tiles<Half, 256, 128, 4, 2>(p.o, p.t, s.slices, stream)
                  : s.bm == 128
                      ? launch_tiles<Half, 128, 128, 2, 2>(p.o, p.t, s.slices, stream)
                      : launch_tiles<Half, 64, 64, 2, 2>(p.o, p.t, s.slices, stream);
    return e != 0 || !p.join ? e : launch_join<Half>(p.t, p.o.M, p.o.N, s.slices, stream);
}

// Two small products in one launch, blockIdx.y the one.
__global__ __launch_bounds__(512) void xent_both_kernel(Operands a, Target to_a, Operands b,
                                                        Target to_b) {
    const bool second = blockIdx.y != 0;
    const Operands o = second ? b : a;
    const int64_t tm = (o.M + 63) / 64, tn = (o.N + 63) / 64;
    if (blockIdx.x >= tm * tn) return;
    Gemm<Half, 64, 64, 2, 2, 4, 2>::run(o, second ? to_b : to_a, tm, tn, 1);
}
bool is_small(const Product& p) { return small(p.o.M, p.o.N, steps_of(p.o.row / 2)); }
int launch_both(const Product& a, const Product& b, void* stream) {
    const int64_t na = up(a.o.M, 64) * up(a.o.N, 64), nb = up(b.o.M, 64) * up(b.o.N, 64);
    return launch(xent_both_kernel, dim3((uint32_t)(na > nb ? na : nb), 2), 512, stream, a.o, a.t,
                  b.o, b.t);
}

struct BackwardRoom : Room {
    int64_t piece, row_ld, class_ld;  // classes of a piece; row lengths of the slopes' parts
    int px, pw;                       // parts
    int64_t by_row, by_class, x, w, largest, ones, rows, classes, sum, slices;
};
// (px: 0 without dx)
BackwardRoom room_of(int64_t T, int64_t V, int64_t K, int px, int pw, int64_t piece) {
    BackwardRoom r;
    r.px = px;
    r.pw = pw;
    r.piece = piece;
    r.row_ld = up(r.piece, kRound) * kRound;
    r.class_ld = up(T, kRound) * kRound;
    r.by_row = r.take(r.px * T * r.row_ld * 2);
    r.by_class = r.take(r.pw * r.piece * r.class_ld * 2);
    r.x = r.take(r.pw * K * r.class_ld * 2);
    r.w = r.take(r.px * K * r.row_ld * 2);
    r.largest = r.take(2 * kLargest * 4);
    r.ones = r.take(K * 4);
    r.rows = r.take(T * 4);
    r.classes = r.take(r.piece * 4);
    const bool pieces = r.piece < V && px > 0;
    if (pieces) r.sum = r.take(T * slices_ld(K) * 4);
    int64_t most = 0;
    const int64_t last = V - (V - 1) / r.piece * r.piece;
    for (int i = 0; i < 2; ++i) {
        const int64_t n = i ? last : r.piece;
        const Shape x = product_shape(T, K, r.px * up(n, kRound));
        const Shape w = product_shape(n, K, r.pw * up(T, kRound));
        const int64_t a = px == 0 ? 0
                          : pieces ? T * slices_ld(K) * 4 * x.slices : slices_bytes(T, K, x);
        const int64_t b = slices_bytes(n, K, w);
        most = a > most ? a : most;
        most = b > most ? b : most;
    }
    r.slices = r.take(most);
    return r;
}
BackwardRoom backward_room(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    const int px = dx_bf16 ? 1 : 2, pw = dw_bf16 ? 1 : 2;
    return room_of(T, V, K, px, pw, piece_of(T, V, K, px));
}
// Without dx, in the room for both: no weights are laid out, and pieces are as large as fit
// (dw alone of 128 x 151936 x 4096 fp32 968 us, in the pieces for both 1054).
BackwardRoom weight_room(const BackwardRoom& both, int64_t T, int64_t V, int64_t K) {
    for (int64_t pieces = up(V, piece_of(T, V)); pieces < up(V, both.piece);
         pieces += 1 + pieces / 8) {
        const BackwardRoom r = room_of(T, V, K, 0, both.pw, piece_size(V, pieces, 256));
        if (r.bytes <= both.bytes) return r;
    }
    return both;
}

// sum <- sum and the slices of a piece, to dx, its rows scaled, after the last piece; 4
// columns a thread
__global__ __launch_bounds__(256) void xent_add_kernel(float* sum, const float* part, int64_t ld,
                                                       int64_t slice, int64_t T, int64_t K,
                                                       int slices, int first, int last,
                                                       const float* rows, Target out) {
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
    const float f = rows[t], v[4] = {x[0] * f, x[1] * f, x[2] * f, x[3] * f};
    store_cols<4>(out, t, k, (int)(K - k < 4 ? K - k : 4), v);
}
int add(const BackwardRoom& r, void* ws, const Loss& l, int slices, bool first, bool last, Mat dx,
        void* stream) {
    Target out{};
    out.ldc = dx.ld;
    out.bf16 = dx.bf16;
    const int64_t ld = slices_ld(l.K), across = up(l.K, 4);
    // (a launch holds fewer than 2^32 work items)
    return in_parts(l.T, across, [&](int64_t t, int64_t n) {
        Target part = out;
        part.c = static_cast<char*>(dx.p) + t * dx.ld * (dx.bf16 ? 2 : 4);
        return launch(xent_add_kernel, dim3((uint32_t)up(n * across, 256)), 256, stream,
                      at<float>(ws, r.sum) + t * ld, at<const float>(ws, r.slices) + t * ld, ld,
                      l.T * ld, n, l.K, slices, (int)first, (int)last,
                      at<const float>(ws, r.rows) + t, part);
    });
}

template <int PX, int PW>
int launch_slopes(const Logits& z, const Slopes& to, int64_t K, void* stream) {
    return with_tile(logit_tile(z.o.M, z.o.N, up(K, kStep), 0, PX + PW).tile, [&](auto tile) {
        const int64_t tm = up(z.o.M, tile), tn = up(z.o.N, tile);
        if (tm * tn * threads(tile) >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
        return launch(xent_slopes_kernel<tile, across(tile), buffers(tile), PX, PW>,
                      dim3((uint32_t)(tm * tn)), threads(tile), stream, z, to, tm, tn);
    });
}

int backward(const Loss& l, const LossIn& in, Mat dx, Mat dw, void* ws, void* stream) {
    const BackwardRoom both = backward_room(l.T, l.V, l.K, dx.bf16, dw.bf16);
    const bool x = dx.p != nullptr, w = dw.p != nullptr;
    const BackwardRoom r = x ? both : weight_room(both, l.T, l.V, l.K);
    const int px = x ? r.px : 0, pw = w ? r.pw : 0;
    auto* turned_x = at<uint16_t>(ws, r.x);
    auto* turned_w = at<uint16_t>(ws, r.w);
    auto* ones = at<float>(ws, r.ones);
    for (int64_t v = 0; v < l.V; v += r.piece) {
        const int64_t n = l.V - v < r.piece ? l.V - v : r.piece;
        const bool first = v == 0, last = v + n == l.V;
        Slopes to{};
        to.by_row = at<uint16_t>(ws, r.by_row);
        to.by_class = at<uint16_t>(ws, r.by_class);
        to.row_ld = up(n, kRound) * kRound;
        to.class_ld = r.class_ld;
        to.in = in;
        to.largest = at<const float>(ws, r.largest);
        to.rows = at<float>(ws, r.rows);
        to.classes = at<float>(ws, r.classes);
        to.V = l.V;
        Source of_x{}, of_w{};
        Largest largest{};
        if (w && first)
            of_x = source(l.x.q, l.x.ld, l.T, l.K, turned_x, r.class_ld, pw);
        if (x) of_w = source(l.w.q + v * l.w.ld, l.w.ld, n, l.K, turned_w, to.row_ld, px);
        if (first) {
            const int64_t parts = up(l.V, kClasses), rows = up(l.T, kTokens);
            const int64_t some = parts > rows ? parts : rows;
            largest = {l.x, l.w, l.target, in.g, l.T, l.V, l.K, at<float>(ws, r.largest), ones,
                       (int)(some < kLargest ? some : kLargest)};
        }
        if (int e = launch_turn(of_x, of_w, largest, stream)) return e;
        const Logits z = logits_of(l, v, n);
        const int e = px == 0   ? pw == 1 ? launch_slopes<0, 1>(z, to, l.K, stream)
                                          : launch_slopes<0, 2>(z, to, l.K, stream)
                      : px == 1 ? pw == 0   ? launch_slopes<1, 0>(z, to, l.K, stream)
                                  : pw == 1 ? launch_slopes<1, 1>(z, to, l.K, stream)
                                            : launch_slopes<1, 2>(z, to, l.K, stream)
                      : pw == 0 ? launch_slopes<2, 0>(z, to, l.K, stream)
                      : pw == 1 ? launch_slopes<2, 1>(z, to, l.K, stream)
                                : launch_slopes<2, 2>(z, to, l.K, stream);
        if (e) return e;
        void* slices = at<char>(ws, r.slices);
        const bool whole = first && last;
        Product for_x{}, for_w{};
        if (x)
            for_x = product_of(to.by_row, turned_w, px * to.row_ld, l.T, l.K, to.rows, ones,
                               whole ? dx : Mat{nullptr, 0, false}, slices);
        if (w)
            for_w = product_of(to.by_class, turned_x, pw * r.class_ld, n, l.K, to.classes, ones,
                               Mat{static_cast<char*>(dw.p) + v * dw.ld * (dw.bf16 ? 2 : 4),
                                   dw.ld, dw.bf16},
                               slices);
        if (x && w && whole && is_small(for_x) && is_small(for_w))
            return launch_both(for_x, for_w, stream);
        if (x) {
            if (int s = launch_product(for_x, stream)) return s;
            if (!whole)
                if (int s = add(r, ws, l, for_x.shape.slices, first, last, dx, stream)) return s;
        }
        if (w)
            if (int s = launch_product(for_w, stream)) return s;
    }
    return 0;
}

template <int TILE>
int few_slopes(const Logits& z, const FewSlopes& to, void* stream) {
    const int64_t tm = up(z.o.M, TILE), tn = up(z.o.N, TILE);
    return launch(xent_few_grads_kernel<TILE, across(TILE), buffers(TILE)>,
                  dim3((uint32_t)(tm * tn)), threads(TILE), stream, z, to, tm, tn);
}

}  // namespace

int64_t xent_workspace(int64_t T, int64_t V, int64_t K) {
    return few_logits(T, K) ? few_xent_workspace(T, V) : forward_room(T, V, K).bytes;
}

int launch_xent(const Loss& l, const LossOut& to, void* workspace, void* stream) {
    return few_logits(l.T, l.K) ? launch_few_xent(l, to, workspace, stream)
                                : forward(l, to, workspace, stream);
}

int launch_few_slopes(const Loss& l, int64_t first, int64_t n, const LossIn& in, float* d,
                      int64_t ld, float* scale, void* stream) {
    const FewSlopes to{d, ld, in, scale, l.V};
    const Logits z = logits_of(l, first, n);
    // (tiles of 256 would be mostly empty)
    return logit_tile(l.T, n, up(l.K, kStep), 0, 1).tile == 64 ? few_slopes<64>(z, to, stream)
                                                               : few_slopes<128>(z, to, stream);
}

int64_t xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    return T <= kFewTokens ? few_xent_bwd_workspace(T, V, K, dx_bf16, dw_bf16)
                           : backward_room(T, V, K, dx_bf16, dw_bf16).bytes;
}

int launch_xent_bwd(const Loss& l, const LossIn& in, Mat dx, Mat dw, void* workspace,
                    void* stream) {
    // a sum over no tokens
    if (l.T == 0)
        return launch_grad_weight(Mat{nullptr, 0, false}, l.x, 0, l.V, l.K, dw, workspace, stream);
    return l.T <= kFewTokens ? launch_few_xent_bwd(l, in, dx, dw, workspace, stream)
                             : backward(l, in, dx, dw, workspace, stream);
}

}  // namespace q8
}  // namespace cpdp
