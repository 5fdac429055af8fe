// Orthogonalised updates: Newton-Schulz iteration of a matrix U, and the weight update that uses it.
//   X <- U / (|U| + eps) with the Frobenius norm;   a step:  A = X X^T,  B = b A + c A A,  X <- a X + B X
// (X^T X and X B for matrices with more rows than columns).  A step maps every singular value s to a s + b s^3 + c s^5 and leaves the
// singular vectors alone.  A and B are symmetric: tiles above their diagonal are computed once and stored twice.
//
// Precision: products on fp16 operands (11 significant bits at bf16's rate; everything here is bounded: |X| by its largest singular value,
// which starts at 1 or less) scaled by powers of two away from fp16's subnormals, sums in fp32.  X itself is kept with 22 bits for the term
// a X, as that operand and what its rounding left, in fp16 too (fp32 beside the operand is two bytes an element more each way) and times 2^11,
// or what is left of elements below 2^-13 would be among fp16's subnormals; below 2^-24, where the operand is, X is kept to 2^-46.
// Small singular values live in that term alone, and an X rounded from step to step would drown them in the rounding of the large ones.
// Where the singular values are close to each other, B is near a multiple of the identity that cancels most of a; that
// multiple, b t + c t t with t the mean of A's diagonal, then goes to the term in fp32 too: X <- (a + shift) X + (B - shift) X.
// (t^2 n > 0.8 |A|^2 says so.  With small singular values among large ones the shifted products would bring the roundings back.)
// Simulated error of the result, 512 x 768 of rank 8: 0.34 with bf16 throughout, 0.04 with fp16, 3e-4 so; full-rank
// Gaussian 64 x 576: 1.2e-2, 1.5e-3, 7e-4 (2e-3 without the shift); Gaussian 27 x 64: 1.3e-3 (2.4e-3 without).
#include <algorithm>
#include <cmath>

#include "tile_product.h"

namespace wap {

namespace {

using namespace tile;

typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kMaxGroup = 16;  // matrices of one set of launches
// what is stored as fp16 times a power of two: X, A = X X^T, B
constexpr float kScaleX = 0x1p10f, kScaleA = 0x1p12f, kScaleB = 0x1p10f, kScaleLow = 0x1p11f;  // (Low: of what X's operand left, once more)

struct Mat {
    int rows, cols, pitch;  // pitch: columns rounded up to 8, zeros behind the last
    int n, npitch;          // the smaller side
    int first;              // first work-group of this matrix in the launch at hand
    bf16_t *x16, *next16;   // [rows][pitch]: X times kScaleX in fp16, of this step and of the next,
    bf16_t* low16;          // ... and what that rounding left
    float* x32;             // few rows: X
    bf16_t *a16, *b16;      // [n][npitch]
    double* parts;          // sums of squares
    float* shift;
    float* sums;     // several work-groups for a few rows: of X X^T, two halves
    f32x2* moments;  // of A's tiles: sums of their diagonal and of their squares
    int nmoments;
    const float* g;
    float* m;    // muon: momentum, master weights and their bf16 copy (NULL: none)
    float* w32;
    bf16_t* w;  // ... or the orthogonal matrix
    float lr, keep;  // keep: 1 - lr * weight decay
    int split;       // parts of the reduction of X X^T
    float* part;     // ... their sums: [tile][part][64][64]
};
enum Way { ONE, MANY, TILES };  // a work-group a matrix and one launch; several of them and a launch a step; products on tiles
struct Group {
    int n, blocks;
    Way way;
    int gram, square, apply;  // tiles of the three products
    bool split;               // X X^T in parts (small tiles)
    Mat mat[kMaxGroup];
};
struct Rule {
    float a, b, c, eps, momentum;
    int nesterov, muon, last;
};

__device__ __forceinline__ int find(const Group& g, int id) {
    int i = 0;
    while (i + 1 < g.n && id >= g.mat[i + 1].first) ++i;
    return i;
}
__device__ __forceinline__ unsigned pack_half2(float a, float b) {
    return (unsigned)__builtin_bit_cast(unsigned short, (_Float16)a) | ((unsigned)__builtin_bit_cast(unsigned short, (_Float16)b) << 16);
}
__device__ __forceinline__ u32x2 pack_half4(f32x4 v) { return u32x2{pack_half2(v[0], v[1]), pack_half2(v[2], v[3])}; }
__device__ __forceinline__ f32x4 unpack_half4(u32x2 p) {
    f32x4 v;
#pragma unroll
    for (int h = 0; h < 4; ++h) v[h] = (float)__builtin_bit_cast(_Float16, (unsigned short)(p[h >> 1] >> (16 * (h & 1))));
    return v;
}

// What a number is multiplied by for a division by a norm: a power of two, then the rest.  In one fp32 number the reciprocal of a norm below
// 2^-128 (momentum that no gradient has reached for long ends there) would be an infinity, of one beyond 2^126 it would lose digits.
struct Divisor {
    float power, rest;
};
__device__ __forceinline__ Divisor divisor(double norm) {
    if (norm == 0.) return {1.f, 0.f};
    // (an infinity, whose exponent is taken as 0, brings finite numbers to 0 and itself, as NaN does everything, to NaN)
    const int e = -__builtin_amdgcn_frexp_exp(norm), power = max(-126, min(126, e));
    return {__builtin_ldexpf(1.f, power), (float)__builtin_ldexp(1. / __builtin_amdgcn_frexp_mant(norm), e - power)};
}
__device__ __forceinline__ float divide(float u, Divisor by) { return u * by.power * by.rest; }

// work-groups of the passes over a matrix: at least 16 elements a thread; of the first one also sums of squares
__host__ __device__ inline int norm_blocks(const Mat& q) {
    const long b = ((long)q.rows * q.cols + 4095) / 4096;
    return b < 256 ? (int)b : 256;
}
__host__ __device__ inline int scale_blocks(const Mat& q) {
    const long b = ((long)q.rows * q.pitch + 4095) / 4096;
    return b < 2048 ? (int)b : 2048;
}

// The update's source: momentum (stored) and the sum of squares of what is to be orthogonalised, in double: one pass, bound by memory
// (121 M elements, FC weights of VGG-16: 280 us, 5.2 TB/s).  A thread adds in its own order, the work-groups' sums are added in order.
__global__ __launch_bounds__(256) void ns_norm_kernel(const Group g, const Rule r) {
    const Mat& q = g.mat[find(g, blockIdx.x)];
    const int block = blockIdx.x - q.first, blocks = norm_blocks(q);
    const long elems = (long)q.rows * q.cols, quads = elems / 4;
    double sum = 0.;
    auto one = [&](float gv, float& mv) {
        float u = gv;
        if (r.muon) {
            mv = __builtin_fmaf(r.momentum, mv, gv);
            u = r.nesterov ? __builtin_fmaf(r.momentum, mv, gv) : mv;
        }
        sum += (double)u * u;
    };
    // (loads of four quads in flight: with one, 4096 x 4096 took 30 us)
    const long stride = (long)blocks * 256;
    for (long i = (long)block * 256 + threadIdx.x; i < quads; i += 4 * stride) {
        f32x4 gv[4], mv[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            gv[u] = mv[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (i + u * stride >= quads) continue;
            gv[u] = reinterpret_cast<const f32x4*>(q.g)[i + u * stride];
            if (r.muon) mv[u] = reinterpret_cast<const f32x4*>(q.m)[i + u * stride];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float t = mv[u][e];
                one(gv[u][e], t);
                mv[u][e] = t;
            }
            if (r.muon && i + u * stride < quads) reinterpret_cast<f32x4*>(q.m)[i + u * stride] = mv[u];
        }
    }
    if (block == 0 && threadIdx.x < (elems & 3)) {
        const long i = quads * 4 + threadIdx.x;
        float mv = r.muon ? q.m[i] : 0.f;
        one(q.g[i], mv);
        if (r.muon) q.m[i] = mv;
    }
    __shared__ double sums[4];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) q.parts[block] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X as its fp16 rounding and the rest
__device__ __forceinline__ void store_x(f32x4 x, u32x2* high, u32x2* low) {
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[e] * kScaleX;
    const u32x2 h = pack_half4(y);
    const f32x4 back = unpack_half4(h);
    *high = h;
    *low = pack_half4(f32x4{(y[0] - back[0]) * kScaleLow, (y[1] - back[1]) * kScaleLow, (y[2] - back[2]) * kScaleLow, (y[3] - back[3]) * kScaleLow});
}

// X of the first step, in rows of whole groups of eight with zeros behind.  (U is computed again rather than stored by the pass before, which
// would move 8 bytes an element more.  FC weights of VGG-16: 285 us, 5.1 TB/s.)
__global__ __launch_bounds__(256) void ns_scale_kernel(const Group g, const Rule r) {
    const Mat& q = g.mat[find(g, blockIdx.x)];
    const int block = blockIdx.x - q.first, blocks = scale_blocks(q), parts = norm_blocks(q);
    const unsigned per = (unsigned)q.pitch / 4, groups = (unsigned)q.rows * per;
    __shared__ double sums[4];
    double sum = threadIdx.x < parts ? q.parts[threadIdx.x] : 0.;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    const Divisor by = divisor(sqrt(sums[0] + sums[1] + sums[2] + sums[3]) + (double)r.eps);
    const bool vec = q.cols % 4 == 0;
    for (unsigned i = block * 256 + threadIdx.x; i < groups; i += blocks * 256) {
        const unsigned row = i / per;
        const int col = (int)(i - row * per) * 4;
        const long at = (long)row * q.cols + col;
        f32x4 u = {0.f, 0.f, 0.f, 0.f}, mv = u;
        if (vec) {
            if (col < q.cols) {
                if (!r.muon || r.nesterov) u = *reinterpret_cast<const f32x4*>(q.g + at);
                if (r.muon) mv = *reinterpret_cast<const f32x4*>(q.m + at);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (col + e >= q.cols) continue;
                if (!r.muon || r.nesterov) u[e] = q.g[at + e];
                if (r.muon) mv[e] = q.m[at + e];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (r.muon) u[e] = r.nesterov ? __builtin_fmaf(r.momentum, mv[e], u[e]) : mv[e];
            u[e] = divide(u[e], by);
        }
        store_x(u, reinterpret_cast<u32x2*>(q.x16) + i, reinterpret_cast<u32x2*>(q.low16) + i);
    }
}

// tile `id` on or below the diagonal of a symmetric matrix of tiles, row by row
__device__ __forceinline__ void triangle(int id, int* row, int* col) {
    int t = (int)((sqrtf(8.f * (float)id + 1.f) - 1.f) * 0.5f);
    while (t * (t + 1) / 2 > id) --t;
    while ((t + 1) * (t + 2) / 2 <= id) ++t;
    *row = t;
    *col = id - t * (t + 1) / 2;
}

// ... in strips of eight rows of tiles, walked column by column: tiles that follow each other share their operands in an XCD's L2
__device__ __forceinline__ void triangle_near(int at, int nt, int* row, int* col) {
    triangle(at, row, col);
    const int first = *row & ~7, high = min(8, nt - first);
    int in = at - first * (first + 1) / 2;
    if (in < (first + 1) * high) {  // columns of the whole strip
        *col = in / high;
        *row = first + in - *col * high;
        return;
    }
    in -= (first + 1) * high;
    int c = 1;  // columns that begin below the strip's first row
    while (in >= high - c) in -= high - c++;
    *col = first + c;
    *row = first + c + in;
}

// from A's trace and sum of squares
__device__ __forceinline__ float shift_of(float trace, float squares, int n, const Rule& r) {
    const float t = trace / (float)n;
    return t * trace > 0.8f * squares ? t * __builtin_fmaf(r.c, t, r.b) : 0.f;
}

// A = X X^T (SQUARE false; X^T X of a tall matrix) or B = b A + c A A (SQUARE true): tiles on and below the diagonal, stored in both orders.
// Bound by the MFMA and, on tiles of 192, by the LDS that feeds it: 4096 x 4096 in 88 us either way, 253 tiles on 256 CUs at 0.87 PFLOP/s
// (with tiles of 256, 136 of them, the whole iteration took 1.70 ms, with these 1.47 at the time); X X^T of the FC weights of VGG-16 515 us, 1.07 PFLOP/s.
template <class W, class T, bool SQUARE>
__global__ __launch_bounds__(W::THREADS, W::THREADS >= 512 ? 2 : 1) void ns_gram_kernel(const Group g, const Rule r) {
    extern __shared__ __align__(16) unsigned char smem[];
    const Mat& q = g.mat[find(g, blockIdx.x)];
    const int nt = (q.n + W::BM - 1) / W::BM, id = of_xcd(blockIdx.x - q.first, nt * (nt + 1) / 2);
    int ti, tj;
    triangle_near(id, nt, &ti, &tj);
    const int m0 = ti * W::BM, n0 = tj * W::BN;
    f32x4 acc[W::FM][W::FN];
    if (SQUARE) {
        const Operand o = {q.a16, q.npitch, q.n, nullptr, 0};
        product<W>(o, o, m0, n0, 0, q.n, smem, acc);
    } else if (q.rows <= q.cols) {
        const Operand o = {q.x16, q.pitch, q.rows, nullptr, 0};
        product<W>(o, o, m0, n0, 0, q.cols, smem, acc);
    } else {
        const Operand o = {q.x16, q.pitch, q.cols, nullptr, 0};
        product<T>(o, o, m0, n0, 0, q.rows, smem, acc);
    }
    bf16_t* out = SQUARE ? q.b16 : q.a16;
    f32x2* meet = reinterpret_cast<f32x2*>(smem);
    auto over_all = [&](f32x2 v) {  // sum over the work-group
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            v[0] += __shfl_xor(v[0], d);
            v[1] += __shfl_xor(v[1], d);
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = v;
        __syncthreads();
        v = f32x2{0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W::WAVES; ++w) {
            v[0] += meet[w][0];
            v[1] += meet[w][1];
        }
        __syncthreads();
        return v;
    };
    float shift = 0.f;  // (of the diagonal: its tiles alone need it)
    if (SQUARE && ti == tj) {
        f32x2 sum = {0.f, 0.f};
        for (int i = threadIdx.x; i < q.nmoments; i += W::THREADS) {
            sum[0] += q.moments[i][0];
            sum[1] += q.moments[i][1];
        }
        sum = over_all(sum);
        shift = shift_of(sum[0], sum[1], q.n, r);
        if (ti == 0 && threadIdx.x == 0) *q.shift = shift;
        shift *= kScaleB;
    }
    f32x2 moments = {0.f, 0.f};
    const float fb = r.b * (kScaleB / kScaleA), fc = r.c * (kScaleB / (kScaleA * kScaleA));
    auto store = [&](int i, int j, f32x4 v) __attribute__((always_inline)) {  // row i, columns j .. j + 3
        if (i < q.n && j < q.npitch) *reinterpret_cast<u32x2*>(out + (size_t)i * q.npitch + j) = pack_half4(v);
    };
    auto ahead = [&](int n, int m) __attribute__((always_inline)) {  // of A
        if constexpr (SQUARE) return *reinterpret_cast<const u32x2*>(q.a16 + (size_t)min(n0 + n, q.n - 1) * q.npitch + min(m0 + m, q.npitch - 4));
        else return Nothing{};
    };
    auto finish = [&](int i, int j, f32x4 v, auto there) __attribute__((always_inline)) {
        f32x4 old = {0.f, 0.f, 0.f, 0.f};
        if constexpr (SQUARE) {
            if (i < q.n && j < q.npitch) old = unpack_half4(there);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = SQUARE ? __builtin_fmaf(fb, old[e], fc * v[e]) - (i == j + e ? shift : 0.f) : v[e] * (kScaleA / (kScaleX * kScaleX));
            if (!SQUARE) {
                const float one = v[e] * (1.f / kScaleA);
                moments[0] += i == j + e ? one : 0.f;
                moments[1] = __builtin_fmaf(one, one, moments[1]);
            }
        }
        store(i, j, v);
        return v;
    };
    // (both orders one after the other, 32 n at a time: the finished values go back into the strip and leave it turned around)
    hand_out<W, true>(acc, smem, ahead, [&](int n, int m, f32x4 v, auto there) { return finish(n0 + n, m0 + m, v, there); },
                      [&](int m, int n, f32x4 v) { if (ti != tj) store(m0 + m, n0 + n, v); });
    if (!SQUARE) {
        moments = over_all(moments);
        if (threadIdx.x == 0) q.moments[id] = f32x2{moments[0], ti == tj ? moments[1] : 2.f * moments[1]};
    }
}

// X X^T of few rows and many columns: parts of the reduction, and their sums in order.  13 filters of VGG-16: 24 and 9 us a step, a chip full
// of short tiles (whole reductions last as long as the longest one: the update of a list with 128 x 11840 took 294 us, with parts 178).
template <class W, class T>
__global__ __launch_bounds__(W::THREADS) void ns_part_kernel(const Group g) {
    extern __shared__ __align__(16) unsigned char smem[];
    // parts are about equally long, so an XCD takes a run of the whole list; the tiles of a part follow each other, they share its columns (13
    // filters of VGG-16: 26 us, 35 with every matrix over all XCDs)
    const int run = of_xcd(blockIdx.x, g.blocks);
    const Mat& q = g.mat[find(g, run)];
    const int nt = (q.n + 63) / 64, all = nt * (nt + 1) / 2, at = run - q.first, part = at / all, id = at - part * all, depth = max(q.rows, q.cols);
    const int per = ((depth + kStep - 1) / kStep + q.split - 1) / q.split * kStep, k0 = part * per, k1 = min(depth, k0 + per);
    int ti, tj;
    triangle_near(id, (q.n + W::BM - 1) / W::BM, &ti, &tj);
    f32x4 acc[W::FM][W::FN];
    if (q.rows <= q.cols) {
        const Operand o = {q.x16, q.pitch, q.rows, nullptr, 0};
        product<W>(o, o, ti * W::BM, tj * W::BN, k0, k1, smem, acc);
    } else {
        const Operand o = {q.x16, q.pitch, q.cols, nullptr, 0};
        product<T>(o, o, ti * W::BM, tj * W::BN, k0, k1, smem, acc);
    }
    f32x4* to = reinterpret_cast<f32x4*>(q.part + ((size_t)id * q.split + part) * (W::BM * W::BN));
    hand_out<W>(acc, smem, [&](int n, int m, f32x4 v) { to[(n * W::BM + m) / 4] = v; });
}
__global__ __launch_bounds__(256) void ns_join_kernel(const Group g) {
    __shared__ float turn[64 * 65];
    __shared__ f32x2 meet[4];
    const Mat& q = g.mat[find(g, blockIdx.x)];
    const int id = blockIdx.x - q.first, t = threadIdx.x;
    int ti, tj;
    triangle_near(id, (q.n + 63) / 64, &ti, &tj);
    f32x2 moments = {0.f, 0.f};
    const f32x4* from = reinterpret_cast<const f32x4*>(q.part + (size_t)id * q.split * 4096);
    f32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = from[k * 256 + t];
    for (int s = 1; s < q.split; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const f32x4 w = from[s * 1024 + k * 256 + t];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k][e] += w[e];
        }
    auto store = [&](int i, int j, f32x4 w) {  // row i, columns j .. j + 3
        if (i < q.n && j < q.npitch) *reinterpret_cast<u32x2*>(q.a16 + (size_t)i * q.npitch + j) = pack_half4(w);
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int n = (k * 256 + t) / 16, m = (t & 15) * 4, i = tj * 64 + n, j = ti * 64 + m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float one = v[k][e] * (1.f / (kScaleX * kScaleX));
            moments[0] += i == j + e ? one : 0.f;
            moments[1] = __builtin_fmaf(one, one, moments[1]);
            v[k][e] *= kScaleA / (kScaleX * kScaleX);
            turn[(m + e) * 65 + n] = v[k][e];
        }
        store(i, j, v[k]);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        moments[0] += __shfl_xor(moments[0], d);
        moments[1] += __shfl_xor(moments[1], d);
    }
    if ((t & 63) == 0) meet[t >> 6] = moments;
    __syncthreads();
    if (t == 0) {
        const float squares = meet[0][1] + meet[1][1] + meet[2][1] + meet[3][1];
        q.moments[id] = f32x2{meet[0][0] + meet[1][0] + meet[2][0] + meet[3][0], ti == tj ? squares : 2.f * squares};
    }
    if (ti == tj) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int m = (k * 256 + t) / 16, n = (t & 15) * 4;
        store(ti * 64 + m, tj * 64 + n, f32x4{turn[m * 65 + n], turn[m * 65 + n + 1], turn[m * 65 + n + 2], turn[m * 65 + n + 3]});
    }
}

// X <- a X + B X (X B of a tall matrix); the last step's goes to where it is used instead.  Products of 4096 steps reach 1.4 PFLOP/s in the
// loop; all CUs then read and write 4 bytes an element of X each way at the same time, a fifth of the whole: 4096 x 4096 in 127 - 141 us,
// 0.97 - 1.08 PFLOP/s; the FC weights of VGG-16 in 1.03 ms (8 rounds of tiles for 7.4); its filters 42 us, bound by X's way (126 MB).
template <class W, class T>
__global__ __launch_bounds__(W::THREADS, W::THREADS >= 512 ? 2 : 1) void ns_apply_kernel(const Group g, const Rule r) {
    extern __shared__ __align__(16) unsigned char smem[];
    const Mat& q = g.mat[find(g, blockIdx.x)];
    int tm, tn;
    tile_of(Tiles{(q.cols + W::BM - 1) / W::BM, (q.rows + W::BN - 1) / W::BN, 8}, blockIdx.x - q.first, &tm, &tn);
    const int m0 = tm * W::BM, n0 = tn * W::BN;
    f32x4 acc[W::FM][W::FN];
    const bf16_t* from = q.x16;
    const float ra = r.a + *q.shift;
    if (q.rows <= q.cols) product<T>(Operand{from, q.pitch, q.cols, nullptr, 0}, Operand{q.b16, q.npitch, q.n, nullptr, 0}, m0, n0, 0, q.n, smem, acc);
    else product<W>(Operand{q.b16, q.npitch, q.n, nullptr, 0}, Operand{from, q.pitch, q.rows, nullptr, 0}, m0, n0, 0, q.n, smem, acc);
    struct Old {
        u32x2 high, low;
        f32x4 w;
    };
    const bool vec = q.cols % 4 == 0, early = r.last && r.muon && vec;
    auto ahead = [&](int n, int m) __attribute__((always_inline)) {
        const size_t at = (size_t)min(n0 + n, q.rows - 1) * q.pitch + min(m0 + m, q.pitch - 4);
        Old x = {*reinterpret_cast<const u32x2*>(q.x16 + at), *reinterpret_cast<const u32x2*>(q.low16 + at), {0.f, 0.f, 0.f, 0.f}};
        if (early) x.w = *reinterpret_cast<const f32x4*>(q.w32 + (size_t)min(n0 + n, q.rows - 1) * q.cols + min(m0 + m, q.cols - 4));
        return x;
    };
    hand_out<W>(acc, smem, ahead, [&](int n, int m, f32x4 v, Old x) __attribute__((always_inline)) {
        n += n0;
        m += m0;
        if (n >= q.rows || m >= q.pitch) return;
        const size_t at = (size_t)n * q.pitch + m;
        const f32x4 high = unpack_half4(x.high), low = unpack_half4(x.low);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(ra * (1.f / kScaleX), __builtin_fmaf(low[e], 1.f / kScaleLow, high[e]), v[e] * (1.f / (kScaleX * kScaleB)));
        if (!r.last) {
            store_x(v, reinterpret_cast<u32x2*>(q.next16 + at), reinterpret_cast<u32x2*>(q.low16 + at));
            return;
        }
        const size_t to = (size_t)n * q.cols + m;
        if (vec && m >= q.cols) return;
        if (r.muon) {
            f32x4 w = x.w;
            if (!vec)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = m + e < q.cols ? q.w32[to + e] : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(-q.lr, v[e], w[e] * q.keep);
            if (vec) *reinterpret_cast<f32x4*>(q.w32 + to) = v;
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (m + e < q.cols) q.w32[to + e] = v[e];
        }
        if (!q.w) return;
        if (vec) *reinterpret_cast<u32x2*>(q.w + to) = pack_bf16x4(v);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (m + e < q.cols) q.w[to + e] = __builtin_bit_cast(unsigned short, (__bf16)v[e]);
    });
}

// ---- matrices of at most 64 rows (columns) ----
// X stays in the registers of eight wavefronts, fp32, each with blocks of 16 columns of all 64 rows (columns and rows of the transposed
// matrix where there are more rows).  In the layout that an MFMA leaves behind (lane: column l & 15, rows 4 (l >> 4) .. + 3 of a block
// of 16) X is, rounded to fp16, the operand of the next B X as it stands, if B's columns are taken in the same order: a reduction may
// run in any.  For X X^T it goes through 4 KB of LDS of the wavefront's own, 32 columns at a time, and comes back transposed.
// Up to 640 columns are one work-group and one launch (five blocks a wavefront; eight do not fit its registers).  More are several work-groups and a launch a step: each finishes A and B of the step by
// itself, from all work-groups' sums of X X^T (10 KB each), applies B to its columns and leaves their sums for the next.
constexpr int kSmallRows = 64, kSmallWaves = 8, kSmallThreads = kSmallWaves * 64;
constexpr int kSmallA = 72;  // elements between rows of A and B: 144 bytes, off each other's banks
constexpr int kSmallTiles = 10, kSmallQuads = kSmallTiles * 64, kSmallStrip = 32 * 144;
constexpr int kSmallSums = kSmallWaves * kSmallTiles * 1024;
constexpr int kSmallLds = kSmallSums + 2 * kSmallRows * kSmallA * 2 + 256;
constexpr int kSmallBlocks[2] = {2, 5};     // of 16 columns a wavefront, at most
constexpr int kManyBlocks = 4;              // ... with several work-groups
constexpr int kManyMost = 64;               // of them: their sums are read by all

__host__ __device__ inline int many_blocks(const Mat& q) { return ((q.rows > q.cols ? q.rows : q.cols) + 16 * kSmallWaves * kManyBlocks - 1) / (16 * kSmallWaves * kManyBlocks); }

template <int BLOCKS>
struct SmallX {
    f32x4 x[BLOCKS][4];
};
__device__ __forceinline__ u32x2 half4(f32x4 v) { return pack_half4(f32x4{v[0] * kScaleX, v[1] * kScaleX, v[2] * kScaleX, v[3] * kScaleX}); }

// Sums of X X^T over the wavefront's columns, tiles (i, j) with j <= i, into the LDS.
template <int BLOCKS>
__device__ __forceinline__ void small_gram(const SmallX<BLOCKS>& s, unsigned char* smem, int wave, int lane) {
    const int l16 = lane & 15, l4 = lane >> 4;
    unsigned char* strip = smem + wave * kSmallTiles * 1024;
    static_assert(kSmallStrip <= kSmallTiles * 1024, "a strip fits the wavefront's sums");
    f32x4 acc[kSmallTiles];
#pragma unroll
    for (int k = 0; k < kSmallTiles; ++k) acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < BLOCKS; b += 2) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // [column][row]
                u32x2 v = {0u, 0u};
                if (b + h < BLOCKS) v = half4(s.x[b + h < BLOCKS ? b + h : b][i]);
                *reinterpret_cast<u32x2*>(strip + (h * 16 + l16) * 144 + (i * 16 + l4 * 4) * 2) = v;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        u32x4 f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned char* p = strip + (l4 * 8 + (l16 >> 2)) * 144 + (i * 16 + (lane & 3) * 4) * 2;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * 144));
            f[i] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j <= i; ++j) acc[i * (i + 1) / 2 + j] = mfma<true>(f[i], f[j], acc[i * (i + 1) / 2 + j]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < kSmallTiles; ++k) *reinterpret_cast<f32x4*>(smem + ((wave * kSmallTiles + k) * 64 + lane) * 16) = acc[k];
    __syncthreads();
}
// Quad k of the wavefronts' sums, added in order.
__device__ __forceinline__ f32x4 small_sum(const unsigned char* smem, int k) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) {
        const f32x4 p = *reinterpret_cast<const f32x4*>(smem + (w * kSmallQuads + k) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += p[e];
    }
    return v;
}
// A step from the finished sums, quad(k) = quad k of kScaleX^2 X X^T: A, B, and X of this wavefront's columns.
template <int BLOCKS, class F>
__device__ __forceinline__ void small_step(SmallX<BLOCKS>& s, const Rule& r, int n, unsigned char* smem, int t, F&& quad) {
    const int lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l16 = lane & 15, l4 = lane >> 4;
    bf16_t* A = reinterpret_cast<bf16_t*>(smem + kSmallSums);
    bf16_t* B = A + kSmallRows * kSmallA;
    f32x2* meet = reinterpret_cast<f32x2*>(B + kSmallRows * kSmallA);
    f32x2 moments = {0.f, 0.f};
#pragma unroll
    for (int turn = 0; turn < (kSmallQuads + kSmallThreads - 1) / kSmallThreads; ++turn) {
        const int k = turn * kSmallThreads + t;
        if (k >= kSmallQuads) break;
        const f32x4 v = quad(k);
        const int tile = k >> 6, i = tile >= 6 ? 3 : tile >= 3 ? 2 : tile >= 1 ? 1 : 0, j = tile - i * (i + 1) / 2;
        const int row = i * 16 + ((k >> 4) & 3) * 4, col = j * 16 + (k & 15);
        u32x2 h = pack_half4(f32x4{v[0] * (kScaleA / (kScaleX * kScaleX)), v[1] * (kScaleA / (kScaleX * kScaleX)), v[2] * (kScaleA / (kScaleX * kScaleX)),
                                   v[3] * (kScaleA / (kScaleX * kScaleX))});
        *reinterpret_cast<u32x2*>(A + col * kSmallA + row) = h;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float one = v[e] * (1.f / (kScaleX * kScaleX));
            moments[0] += row + e == col ? one : 0.f;
            moments[1] = __builtin_fmaf(i == j ? one : 2.f * one, one, moments[1]);
            if (i != j) A[(row + e) * kSmallA + col] = (unsigned short)(h[e >> 1] >> (16 * (e & 1)));
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        moments[0] += __shfl_xor(moments[0], d);
        moments[1] += __shfl_xor(moments[1], d);
    }
    if (lane == 0) meet[wave] = moments;
    __syncthreads();
    moments = f32x2{0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) {
        moments[0] += meet[w][0];
        moments[1] += meet[w][1];
    }
    const float shift = shift_of(moments[0], moments[1], n, r);
    // B: two tiles a wavefront
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = wave >> 1, j = (wave & 1) * 2 + k;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
            v = mfma<true>(*reinterpret_cast<const u32x4*>(A + (i * 16 + l16) * kSmallA + h * 32 + l4 * 8), *reinterpret_cast<const u32x4*>(A + (j * 16 + l16) * kSmallA + h * 32 + l4 * 8), v);
        // rows i * 16 + l4 * 4 + e, column j * 16 + l16: stored at the mirrored place, four columns of a row
        const int row = j * 16 + l16, col = i * 16 + l4 * 4;
        const f32x4 old = unpack_half4(*reinterpret_cast<const u32x2*>(A + row * kSmallA + col));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = __builtin_fmaf(r.b * (kScaleB / kScaleA), old[e], r.c * (kScaleB / (kScaleA * kScaleA)) * v[e]) - (row == col + e && row < n ? shift * kScaleB : 0.f);
        *reinterpret_cast<u32x2*>(B + row * kSmallA + col) = pack_half4(v);
    }
    __syncthreads();
    // X: B's columns in the order in which a lane has X's rows
    u32x4 fb[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bf16_t* p = B + (i * 16 + l16) * kSmallA + h * 32 + l4 * 4;
            const u32x2 lo = *reinterpret_cast<const u32x2*>(p), hi = *reinterpret_cast<const u32x2*>(p + 16);
            fb[i][h] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        u32x4 fx[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x2 lo = half4(s.x[b][2 * h]), hi = half4(s.x[b][2 * h + 1]);
            fx[h] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int h = 0; h < 2; ++h) v = mfma<true>(fb[i][h], fx[h], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) s.x[b][i][e] = __builtin_fmaf(r.a + shift, s.x[b][i][e], v[e] * (1.f / (kScaleX * kScaleB)));
        }
    }
}
// Places in the caller's matrices of this lane's values of block b, and which exist; c0: the work-group's first column.  A value that does
// not exist has the place of the first one: loads need no branch, and a block's are all under way at a time.
struct SmallPlaces {
    unsigned at[4][4];
    unsigned there;  // a bit for each
    __device__ __forceinline__ SmallPlaces(const Mat& q, int c0, int b, int wave, int lane) {
        const bool tall = q.rows > q.cols;
        const int n = min(q.rows, q.cols), m = max(q.rows, q.cols), row0 = (lane >> 4) * 4, col = c0 + (wave + b * kSmallWaves) * 16 + (lane & 15);
        const unsigned along = tall ? 1 : q.cols, first = (unsigned)col * (tall ? q.cols : 1);  // from row to row of the wide matrix
        there = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = row0 + i * 16 + e;
                const bool is = row < n && col < m;
                at[i][e] = is ? row * along + first : 0u;
                there |= is ? 1u << (i * 4 + e) : 0u;
            }
    }
    __device__ __forceinline__ bool has(int i, int e) const { return there >> (i * 4 + e) & 1u; }
};
#define SMALL_ALL _Pragma("unroll") for (int i = 0; i < 4; ++i) _Pragma("unroll") for (int e = 0; e < 4; ++e)
template <int BLOCKS>
__device__ __forceinline__ void small_read(SmallX<BLOCKS>& s, const Mat& q, const Rule& r, int c0, int wave, int lane) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        const SmallPlaces p(q, c0, b, wave, lane);
        f32x4(&x)[4] = s.x[b];
        SMALL_ALL x[i][e] = q.g[p.at[i][e]];
        if (r.muon) {
            float old[4][4];
            SMALL_ALL old[i][e] = q.m[p.at[i][e]];
            SMALL_ALL {
                const float g = x[i][e], mv = __builtin_fmaf(r.momentum, old[i][e], g);
                if (p.has(i, e)) q.m[p.at[i][e]] = mv;
                x[i][e] = r.nesterov ? __builtin_fmaf(r.momentum, mv, g) : mv;
            }
        }
        SMALL_ALL x[i][e] = p.has(i, e) ? x[i][e] : 0.f;
        __builtin_amdgcn_sched_barrier(0);
    }
}
template <int BLOCKS>
__device__ __forceinline__ void small_write(SmallX<BLOCKS>& s, const Mat& q, const Rule& r, int c0, int wave, int lane) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        __builtin_amdgcn_sched_barrier(0);
        const SmallPlaces p(q, c0, b, wave, lane);
        f32x4(&x)[4] = s.x[b];
        if (r.muon) {
            float old[4][4];
            SMALL_ALL old[i][e] = q.w32[p.at[i][e]];
            SMALL_ALL {
                x[i][e] = __builtin_fmaf(-q.lr, x[i][e], old[i][e] * q.keep);
                if (p.has(i, e)) q.w32[p.at[i][e]] = x[i][e];
            }
        }
        if (q.w) SMALL_ALL if (p.has(i, e)) q.w[p.at[i][e]] = __builtin_bit_cast(unsigned short, (__bf16)x[i][e]);
    }
}
#undef SMALL_ALL
template <int BLOCKS>
__device__ __forceinline__ double small_squares(const SmallX<BLOCKS>& s, double* meet, int wave, int lane) {
    double square = 0.;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) square = __builtin_fma((double)s.x[b][i][e], (double)s.x[b][i][e], square);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) square += __shfl_xor(square, d);
    if (lane == 0) meet[wave] = square;
    __syncthreads();
    square = 0.;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) square += meet[w];
    return square;
}
template <int BLOCKS>
__device__ __forceinline__ void small_divide(SmallX<BLOCKS>& s, Divisor by) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s.x[b][i][e] = divide(s.x[b][i][e], by);
}

// All of a matrix in one work-group: X in the registers, A and B in the LDS, every step behind the other without a launch.  64 x 576 with
// five steps takes 34 us (in 17 launches: 69): 4.5 a step, bound by its chain of sums through the LDS, dependent products and barriers,
// and 11 for the launch, the loads (a block of columns waits for the one before), the norm and the stores.
template <int BLOCKS>
__global__ __launch_bounds__(kSmallThreads, 2) void ns_small_kernel(const Group g, const Rule r, int steps) {
    extern __shared__ __align__(16) unsigned char smem[];
    const Mat& q = g.mat[blockIdx.x];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), n = min(q.rows, q.cols);
    SmallX<BLOCKS> s;
    small_read(s, q, r, 0, wave, lane);
    small_divide(s, divisor(sqrt(small_squares(s, reinterpret_cast<double*>(smem + kSmallLds - 256), wave, lane)) + (double)r.eps));
    for (int k = 0; k < steps; ++k) {
        small_gram(s, smem, wave, lane);
        small_step(s, r, n, smem, t, [&](int at) { return small_sum(smem, at); });
    }
    small_write(s, q, r, 0, wave, lane);
}

// Several work-groups a matrix, a launch a step.  step 0: the update's source, its squares, and X X^T of each work-group's columns divided
// by their own norm; then the steps 1 .. steps.  x32, parts and sums hold what lasts from launch to launch.
__global__ __launch_bounds__(kSmallThreads, 2) void ns_many_kernel(const Group g, const Rule r, int step) {
    extern __shared__ __align__(16) unsigned char smem[];
    const Mat& q = g.mat[find(g, blockIdx.x)];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), n = min(q.rows, q.cols);
    const int block = blockIdx.x - q.first, blocks = many_blocks(q), c0 = block * 16 * kSmallWaves * kManyBlocks;
    double* meet = reinterpret_cast<double*>(smem + kSmallLds - 256);
    f32x4* x32 = reinterpret_cast<f32x4*>(q.x32) + (size_t)block * kManyBlocks * 4 * kSmallThreads + t;
    f32x4* sums = reinterpret_cast<f32x4*>(q.sums) + (step & 1) * blocks * kSmallQuads;  // of this step; the other half: the next one's
    SmallX<kManyBlocks> s;
    double square = 0.;
    if (step == 0) {
        small_read(s, q, r, c0, wave, lane);
        square = small_squares(s, meet, wave, lane);
        if (t == 0) q.parts[block] = square;
    } else {
#pragma unroll
        for (int b = 0; b < kManyBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) s.x[b][i] = x32[(b * 4 + i) * kSmallThreads];
        if (step == 1) {
            for (int p = 0; p < blocks; ++p) square += q.parts[p];
            const double norm = sqrt(square) + (double)r.eps;
            small_divide(s, divisor(norm));
            // (a share of the columns without any entry has no norm and no sums; one next to nothing has finite sums and a share of 0)
            small_step(s, r, n, smem, t, [&](int k) {
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
                for (int p = 0; p < blocks; ++p) {
                    const f32x4 w = sums[p * kSmallQuads + k];
                    const float share = norm == 0. ? 0.f : (float)(q.parts[p] / norm / norm);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(share, w[e], v[e]);
                }
                return v;
            });
        } else {
            small_step(s, r, n, smem, t, [&](int k) {
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
                for (int p = 0; p < blocks; ++p) {
                    const f32x4 w = sums[p * kSmallQuads + k];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += w[e];
                }
                return v;
            });
        }
        if (r.last) {
            small_write(s, q, r, c0, wave, lane);
            return;
        }
    }
#pragma unroll
    for (int b = 0; b < kManyBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) x32[(b * 4 + i) * kSmallThreads] = s.x[b][i];
    if (step == 0) small_divide(s, divisor(sqrt(square)));
    small_gram(s, smem, wave, lane);
    f32x4* next = reinterpret_cast<f32x4*>(q.sums) + ((step + 1) & 1) * blocks * kSmallQuads + (size_t)block * kSmallQuads;
    for (int k = t; k < kSmallQuads; k += kSmallThreads) next[k] = small_sum(smem, k);
}

// The tiles: k-rows and i-rows of the M and of the N operand.
template <bool M_IROWS, bool N_IROWS>
using Large = Shape<256, 256, 2, 4, 2, M_IROWS, N_IROWS, true>;
template <bool M_IROWS, bool N_IROWS>
using Medium = Shape<128, 128, 2, 2, 4, M_IROWS, N_IROWS, true>;
template <bool M_IROWS, bool N_IROWS>
using Middle = Shape<192, 192, 4, 2, 3, M_IROWS, N_IROWS, true>;
template <bool M_IROWS, bool N_IROWS>
using Small = Shape<64, 64, 2, 2, 4, M_IROWS, N_IROWS, true>;

template <class S>
int launch(void (*kernel)(Group, Rule), const Group& g, const Rule& r, const char* what, hipStream_t st, std::atomic<bool>& allowed) {
    if (!allowed) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) return set_error(WAP_EHIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
        allowed = true;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)g.blocks), dim3(S::THREADS), S::LDS, st, g, r);
    return check_launch(what);
}
template <template <bool, bool> class S, bool SQUARE>
int launch_gram(const Group& g, const Rule& r, hipStream_t st) {
    static std::atomic<bool> allowed{false};
    return launch<S<false, false>>((void (*)(Group, Rule))ns_gram_kernel<S<false, false>, S<true, true>, SQUARE>, g, r, SQUARE ? "ns_square" : "ns_gram", st, allowed);
}
template <template <bool, bool> class S>
int launch_apply(const Group& g, const Rule& r, hipStream_t st) {
    static std::atomic<bool> allowed{false};
    return launch<S<false, false>>((void (*)(Group, Rule))ns_apply_kernel<S<false, false>, S<true, false>>, g, r, "ns_apply", st, allowed);
}

template <class F>
void number(Group& g, F&& blocks) {  // first work-groups of a launch
    g.blocks = 0;
    for (int i = 0; i < g.n; ++i) {
        g.mat[i].first = g.blocks;
        g.blocks += blocks(g.mat[i]);
    }
}
int tiles_across(int n, int tile) { return (n + tile - 1) / tile; }

int squares(const Mat& q, int tile) {
    const int t = tiles_across(q.n, tile);
    return t * (t + 1) / 2;
}
int whole(const Mat& q, int tile) { return tiles_across(q.rows, tile) * tiles_across(q.cols, tile); }

// How a group runs.
void plan(Group& g) {
    // Matrices of few rows take one launch, or one a step; beside a larger one they ride along in its launches for nothing.
    int columns = 0, groups = 0;
    bool few = true;
    for (int i = 0; i < g.n; ++i) {
        few = few && g.mat[i].n <= kSmallRows;
        columns = std::max(columns, std::max(g.mat[i].rows, g.mat[i].cols));
        groups = std::max(groups, many_blocks(g.mat[i]));
    }
    g.way = few && columns <= kSmallBlocks[1] * 16 * kSmallWaves ? ONE : few && groups <= kManyMost ? MANY : TILES;
    if (g.way != TILES) return;
    // Which tile: the work on the fullest CU (X X^T at 512 x 4608 takes 99 / 41 / 18 us on tiles of 256 / 128 / 64, at 2048 x 2048
    // 55 / 26 / 24, at 4096 x 4096 102 / 120 / 149).
    auto pick = [&](auto&& tiles, auto&& depth, bool store, double* us_out) {
        static const double beside[2][4] = {{8., 5., 1.5, 7.}, {20., 9., 3., 14.}};
        int best = 0;
        double least = 0.;
        for (int k = 0; k < 4; ++k) {
            double count = 0., longest = 0., sum = 0., long_ones = 0., us = 0.;
            for (int i = 0; i < g.n; ++i) count += tiles(g.mat[i], kSides[k]);
            auto one = [&](int i) { return tile_us(k, count, (depth(g.mat[i]) + 63) / 64, beside[store]); };
            for (int i = 0; i < g.n; ++i) {
                longest = std::max(longest, one(i));
                sum += tiles(g.mat[i], kSides[k]) * one(i);
                if (k == 2) us = std::max(us, last_small_tile_us((depth(g.mat[i]) + 63) / 64, count));
            }
            // (tiles that take about as long as the longest go through the CUs in whole rounds)
            for (int i = 0; i < g.n; ++i) long_ones += one(i) >= 0.7 * longest ? tiles(g.mat[i], kSides[k]) : 0;
            us = std::max(us, k == 2 ? sum / kNumCU : std::max(std::ceil(long_ones / kNumCU) * longest, sum / kNumCU));
            if (k == 0 || us < least) { best = k; least = us; }
        }
        *us_out = least;
        return best;
    };
    double us = 0., other = 0.;
    auto longer = [](const Mat& q) { return std::max(q.rows, q.cols); };
    auto shorter = [](const Mat& q) { return q.n; };
    g.gram = pick(squares, longer, false, &us);
    g.square = pick(squares, shorter, false, &other);
    g.apply = pick(whole, shorter, true, &other);
    // X X^T in parts of so many stages, where a second launch is less than what that saves (30 x 15619 and 128 x 11840: 41 to 54 us whole)
    g.split = false;
    int best = 0;
    for (int stages : {8, 12, 16, 24, 32, 48, 64}) {
        static const double beside[4] = {8., 5., 1.5, 7.};
        double sum = 0., bytes = 0., units = 0.;
        for (int i = 0; i < g.n; ++i) {
            const int all = tiles_across(longer(g.mat[i]), kStep), parts = std::min(32, tiles_across(all, stages));
            sum += (double)squares(g.mat[i], 64) * parts * tile_us(2, 1., tiles_across(all, parts), beside);
            units += (double)squares(g.mat[i], 64) * parts;
            bytes += (double)squares(g.mat[i], 64) * parts * 16384.;
        }
        const double t = std::max(sum / kNumCU, last_small_tile_us(stages, units)) + 4. + bytes * 2. / 4e6;
        if (bytes <= 64e6 && t < us) { us = t; best = stages; }
    }
    for (int i = 0; i < g.n; ++i) g.mat[i].split = 1;
    if (best) {
        g.split = true;
        g.gram = 2;
        for (int i = 0; i < g.n; ++i) g.mat[i].split = std::min(32, tiles_across(tiles_across(longer(g.mat[i]), kStep), best));
    }
}

size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
// Lays a matrix's scratch out behind `at`, as far as its group's way needs it (one work-group: nothing lies in memory); base == NULL: only its size.
size_t place(Mat& q, const Group& g, unsigned char* base, size_t at) {
    auto take = [&](size_t bytes) {
        unsigned char* p = base ? base + at : nullptr;
        at += up256(bytes);
        return p;
    };
    q.parts = (double*)take(256 * sizeof(double));
    if (g.way == MANY) {
        const size_t groups = (size_t)many_blocks(q);
        q.x32 = (float*)take(groups * kManyBlocks * kSmallThreads * 4 * sizeof(f32x4));
        q.sums = (float*)take(2 * groups * kSmallQuads * sizeof(f32x4));
    }
    if (g.way == TILES) {
        const size_t elems = (size_t)q.rows * q.pitch, square = (size_t)q.n * q.npitch, tiles = (size_t)(q.n + 63) / 64;
        q.shift = (float*)take(4);
        q.moments = (f32x2*)take(tiles * (tiles + 1) / 2 * sizeof(f32x2));
        q.low16 = (bf16_t*)take(elems * 2);
        q.x16 = (bf16_t*)take(elems * 2);
        q.next16 = (bf16_t*)take(elems * 2);
        q.a16 = (bf16_t*)take(square * 2);
        q.b16 = (bf16_t*)take(square * 2);
        if (g.split) q.part = (float*)take((size_t)squares(q, 64) * q.split * 4096 * sizeof(float));
    }
    return at;
}

int validate_size(int32_t rows, int32_t cols, int i) {
    if (rows < 1 || cols < 1) return set_error(WAP_EINVAL, "matrix %d: every size must be >= 1 (rows=%d cols=%d)", i, rows, cols);
    if (rows > (1 << 24) || cols > (1 << 20) || (long long)rows * ((cols + 7) & ~7) > (1LL << 33))
        return set_error(WAP_EUNSUPPORTED, "matrix %d: more than 2^24 rows, 2^20 columns or 2^33 elements (rows=%d cols=%d)", i, rows, cols);
    return WAP_OK;
}
int validate_ns(const wap_ns_desc& d) {
    if (d.steps < 1 || d.steps > 100) return set_error(WAP_EINVAL, "newton-schulz: steps must be 1 .. 100 (%d)", d.steps);
    if (!std::isfinite(d.a) || !std::isfinite(d.b) || !std::isfinite(d.c)) return set_error(WAP_EINVAL, "newton-schulz: a, b and c must be finite");
    if (!(d.eps >= 0.f) || !std::isfinite(d.eps)) return set_error(WAP_EINVAL, "newton-schulz: eps must be >= 0 and finite");
    return WAP_OK;
}
int check(const void* p, const char* name, int i) {
    if (!p) return set_error(WAP_EINVAL, "matrix %d: %s is NULL", i, name);
    if (reinterpret_cast<uintptr_t>(p) & 15u) return set_error(WAP_EINVAL, "matrix %d: %s is not 16-byte aligned", i, name);
    return WAP_OK;
}

template <int BLOCKS>
int launch_small(const Group& g, const Rule& r, int steps, hipStream_t st) {
    static std::atomic<bool> allowed{false};
    if (!allowed) {
        const hipError_t e = hipFuncSetAttribute((const void*)ns_small_kernel<BLOCKS>, hipFuncAttributeMaxDynamicSharedMemorySize, kSmallLds);
        if (e != hipSuccess) return set_error(WAP_EHIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
        allowed = true;
    }
    hipLaunchKernelGGL(ns_small_kernel<BLOCKS>, dim3((unsigned)g.n), dim3(kSmallWaves * 64), kSmallLds, st, g, r, steps);
    return check_launch("ns_small");
}

int launch_part(const Group& g, hipStream_t st) {
    typedef Small<false, false> S;
    static std::atomic<bool> allowed{false};
    const auto kernel = ns_part_kernel<S, Small<true, true>>;
    if (!allowed) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) return set_error(WAP_EHIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
        allowed = true;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)g.blocks), dim3(S::THREADS), S::LDS, st, g);
    return check_launch("ns_part");
}

int run_group(Group& g, Rule r, int steps, hipStream_t st) {
    int rc;
    if (g.way == ONE) {
        int most = 0;
        for (int i = 0; i < g.n; ++i) most = std::max(most, tiles_across(std::max(g.mat[i].rows, g.mat[i].cols), 16 * kSmallWaves));
        return most <= kSmallBlocks[0] ? launch_small<kSmallBlocks[0]>(g, r, steps, st) : launch_small<kSmallBlocks[1]>(g, r, steps, st);
    }
    if (g.way == MANY) {
        static std::atomic<bool> allowed{false};
        if (!allowed) {
            const hipError_t e = hipFuncSetAttribute((const void*)ns_many_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kSmallLds);
            if (e != hipSuccess) return set_error(WAP_EHIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
            allowed = true;
        }
        number(g, many_blocks);
        for (int s = 0; s <= steps; ++s) {
            r.last = s == steps;
            hipLaunchKernelGGL(ns_many_kernel, dim3((unsigned)g.blocks), dim3(kSmallThreads), kSmallLds, st, g, r, s);
            if ((rc = check_launch("ns_many")) != WAP_OK) return rc;
        }
        return WAP_OK;
    }
    number(g, norm_blocks);
    hipLaunchKernelGGL(ns_norm_kernel, dim3((unsigned)g.blocks), dim3(256), 0, st, g, r);
    if ((rc = check_launch("ns_norm")) != WAP_OK) return rc;
    number(g, scale_blocks);
    hipLaunchKernelGGL(ns_scale_kernel, dim3((unsigned)g.blocks), dim3(256), 0, st, g, r);
    if ((rc = check_launch("ns_scale")) != WAP_OK) return rc;
    for (int i = 0; i < g.n; ++i) g.mat[i].nmoments = squares(g.mat[i], kSides[g.gram]);
    for (int s = 0; s < steps; ++s) {
        r.last = s + 1 == steps;
        if (g.split) {
            number(g, [](const Mat& q) { return squares(q, 64) * q.split; });
            if ((rc = launch_part(g, st)) != WAP_OK) return rc;
            number(g, [](const Mat& q) { return squares(q, 64); });
            hipLaunchKernelGGL(ns_join_kernel, dim3((unsigned)g.blocks), dim3(256), 0, st, g);
            rc = check_launch("ns_join");
        } else {
            number(g, [&](const Mat& q) { return squares(q, kSides[g.gram]); });
            rc = g.gram == 0 ? launch_gram<Large, false>(g, r, st) : g.gram == 1 ? launch_gram<Medium, false>(g, r, st)
               : g.gram == 2 ? launch_gram<Small, false>(g, r, st) : launch_gram<Middle, false>(g, r, st);
        }
        if (rc != WAP_OK) return rc;
        number(g, [&](const Mat& q) { return squares(q, kSides[g.square]); });
        rc = g.square == 0 ? launch_gram<Large, true>(g, r, st) : g.square == 1 ? launch_gram<Medium, true>(g, r, st)
           : g.square == 2 ? launch_gram<Small, true>(g, r, st) : launch_gram<Middle, true>(g, r, st);
        if (rc != WAP_OK) return rc;
        number(g, [&](const Mat& q) { return whole(q, kSides[g.apply]); });
        rc = g.apply == 0 ? launch_apply<Large>(g, r, st) : g.apply == 1 ? launch_apply<Medium>(g, r, st)
           : g.apply == 2 ? launch_apply<Small>(g, r, st) : launch_apply<Middle>(g, r, st);
        if (rc != WAP_OK) return rc;
        for (int i = 0; i < g.n; ++i) std::swap(g.mat[i].x16, g.mat[i].next16);
    }
    return WAP_OK;
}

// The next matrices of the list from *i on, their plan and their places behind `base` (NULL: only the size).
template <class F>
Group next_group(int n, int* i, unsigned char* base, size_t* bytes, F&& at) {
    Group g = {};
    for (; g.n < kMaxGroup && *i < n; ++*i) {
        Mat& q = g.mat[g.n++];
        at(*i, q);
        q.pitch = (q.cols + 7) & ~7;
        q.n = std::min(q.rows, q.cols);
        q.npitch = (q.n + 7) & ~7;
    }
    plan(g);
    *bytes = 0;
    for (int k = 0; k < g.n; ++k) *bytes = place(g.mat[k], g, base, *bytes);
    return g;
}
template <class F>
size_t workspace(int n, F&& at) {
    size_t most = 0, bytes = 0;
    for (int i = 0; i < n; most = std::max(most, bytes)) next_group(n, &i, nullptr, &bytes, at);
    return most;
}
template <class F>
int run(int n, const wap_ns_desc& d, Rule r, void* ws, size_t ws_bytes, hipStream_t st, F&& at) {
    const size_t need = workspace(n, at);
    if (!ws || ws_bytes < need) return set_error(WAP_EWORKSPACE, "newton-schulz: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return set_error(WAP_EINVAL, "workspace is not 256-byte aligned");
    r.a = d.a; r.b = d.b; r.c = d.c; r.eps = d.eps;
    for (int i = 0; i < n;) {
        size_t bytes = 0;
        Group g = next_group(n, &i, (unsigned char*)ws, &bytes, at);
        const int rc = run_group(g, r, d.steps, st);
        if (rc != WAP_OK) return rc;
    }
    return WAP_OK;
}
void fill(const wap_ns_matrix& a, Mat& q) {
    q.rows = a.rows; q.cols = a.cols;
    q.g = a.g;
    q.w = (bf16_t*)a.o;
}
void fill(const wap_muon_matrix& a, float decay, Mat& q) {
    q.rows = a.rows; q.cols = a.cols;
    q.g = a.g; q.m = a.m; q.w32 = a.w32;
    q.w = (bf16_t*)a.w_bf16;
    q.lr = a.lr;
    q.keep = 1.f - a.lr * decay;
}

}  // namespace

}  // namespace wap

using namespace wap;

#define NS_TRY(expr)                   \
    do {                               \
        const int rc_ = (expr);        \
        if (rc_ != WAP_OK) return rc_; \
    } while (0)

static int check_list(const void* mats, int32_t n) {
    if (!mats) return set_error(WAP_EINVAL, "the list of matrices is NULL");
    if (n < 1) return set_error(WAP_EINVAL, "the list of matrices must have at least one (%d)", n);
    return WAP_OK;
}
static int check_sizes(const wap_ns_matrix* mats, int32_t n) {
    NS_TRY(check_list(mats, n));
    for (int i = 0; i < n; ++i) NS_TRY(validate_size(mats[i].rows, mats[i].cols, i));
    return WAP_OK;
}
static int check_sizes(const wap_muon_matrix* mats, int32_t n) {
    NS_TRY(check_list(mats, n));
    for (int i = 0; i < n; ++i) NS_TRY(validate_size(mats[i].rows, mats[i].cols, i));
    return WAP_OK;
}

extern "C" {

int wap_orthogonalise_workspace_bytes(const wap_ns_desc* d, const wap_ns_matrix* mats, int32_t n, size_t* bytes_out) {
    if (!d || !bytes_out) return set_error(WAP_EINVAL, "newton-schulz: NULL argument");
    NS_TRY(validate_ns(*d));
    NS_TRY(check_sizes(mats, n));
    *bytes_out = workspace(n, [&](int i, Mat& q) { fill(mats[i], q); });
    return WAP_OK;
}

int wap_orthogonalise(const wap_ns_desc* d, const wap_ns_matrix* mats, int32_t n, void* ws, size_t ws_bytes, void* stream) {
    if (!d) return set_error(WAP_EINVAL, "newton-schulz descriptor is NULL");
    NS_TRY(validate_ns(*d));
    NS_TRY(check_sizes(mats, n));
    for (int i = 0; i < n; ++i) {
        NS_TRY(check(mats[i].g, "g", i));
        NS_TRY(check(mats[i].o, "o", i));
    }
    return run(n, *d, Rule{}, ws, ws_bytes, (hipStream_t)stream, [&](int i, Mat& q) { fill(mats[i], q); });
}

int wap_muon_workspace_bytes(const wap_muon_desc* d, const wap_muon_matrix* mats, int32_t n, size_t* bytes_out) {
    if (!d || !bytes_out) return set_error(WAP_EINVAL, "muon: NULL argument");
    NS_TRY(validate_ns(d->ns));
    NS_TRY(check_sizes(mats, n));
    *bytes_out = workspace(n, [&](int i, Mat& q) { fill(mats[i], 0.f, q); });
    return WAP_OK;
}

int wap_muon_update(const wap_muon_desc* d, const wap_muon_matrix* mats, int32_t n, void* ws, size_t ws_bytes, void* stream) {
    if (!d) return set_error(WAP_EINVAL, "muon descriptor is NULL");
    NS_TRY(validate_ns(d->ns));
    if (d->flags & ~WAP_MUON_NESTEROV) return set_error(WAP_EINVAL, "muon descriptor: unknown flag bits 0x%x", d->flags);
    if (!(d->momentum >= 0.f) || !std::isfinite(d->momentum)) return set_error(WAP_EINVAL, "muon: momentum must be >= 0 and finite");
    if (!std::isfinite(d->weight_decay)) return set_error(WAP_EINVAL, "muon: weight_decay must be finite");
    NS_TRY(check_sizes(mats, n));
    for (int i = 0; i < n; ++i) {
        NS_TRY(check(mats[i].w32, "w32", i));
        NS_TRY(check(mats[i].m, "m", i));
        NS_TRY(check(mats[i].g, "g", i));
        if (mats[i].w_bf16) NS_TRY(check(mats[i].w_bf16, "w_bf16", i));
        if (!std::isfinite(mats[i].lr)) return set_error(WAP_EINVAL, "matrix %d: lr must be finite", i);
    }
    Rule r = {};
    r.muon = 1;
    r.momentum = d->momentum;
    r.nesterov = (d->flags & WAP_MUON_NESTEROV) != 0;
    return run(n, d->ns, r, ws, ws_bytes, (hipStream_t)stream, [&](int i, Mat& q) { fill(mats[i], d->weight_decay, q); });
}

}  // extern "C"
