// Softmax cross-entropy of features under a classifier's weights, the product included, without the logits of a large product in memory:
//   z = x W^T,  row_loss[n] = log sum over v of exp z[n][v] - z[n][label n],  loss = mean over the rows that have a label,
//   dz = (softmax z - one-hot) * scale / rows with a label,  dx = dz W,  dW = dz^T x.
#include <algorithm>
#include <cmath>

#include "tile_product.h"

namespace wap {

namespace {

using namespace tile;

constexpr float kLog2e = 1.44269504088896340736f;

// What the sums of a row come to in two steps: (largest logit, sum of exp(z - largest)) of some of its classes, and their union.
struct Part {
    float most, sum;
};
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// A row's softmax is exp2((z - most) log2 e - log2 of the sum): with the logarithm of the whole sum of exponentials in one number, a row that is
// sure of its class would round p - 1 to what a logit of 20 rounds to, 2e-6, and its loss to below zero.
struct Norm {
    float most, log2_sum;
};
__device__ __forceinline__ float softmax_of(float z, Norm n) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z - n.most, kLog2e, -n.log2_sum)); }
__device__ __forceinline__ Part join(Part a, Part b) {
    const float most = fmaxf(a.most, b.most);
    // (nothing but -inf on one side: its sum is 0 and stays so)
    const float sa = a.most == -INFINITY ? a.sum : a.sum * exp_of(a.most - most), sb = b.most == -INFINITY ? b.sum : b.sum * exp_of(b.most - most);
    return {most, sa + sb};
}

// Mean of the rows that count, in a fixed order, by one work-group of THREADS.
template <int THREADS>
__device__ __forceinline__ void mean_of(const float* row_loss, const int32_t* labels, int rows, int classes, float* loss) {
    __shared__ double sums[THREADS / 64];
    __shared__ int counts[THREADS / 64];
    double sum = 0.;
    int count = 0;
    for (int n = threadIdx.x; n < rows; n += THREADS) {
        if ((unsigned)labels[n] < (unsigned)classes) {
            sum += row_loss[n];
            ++count;
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        sum += __shfl_xor(sum, d);
        count += __shfl_xor(count, d);
    }
    if ((threadIdx.x & 63) == 0) {
        sums[threadIdx.x >> 6] = sum;
        counts[threadIdx.x >> 6] = count;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS / 64; ++w) {
            sum += sums[w];
            count += counts[w];
        }
        *loss = count ? (float)(sum / count) : 0.f;
    }
}

enum Mode { STATS, STATS_KEEP, PARTIAL, GRAD };

struct XentArgs {
    Operand w, x;  // [classes][features], [rows][features]
    Tiles tiles;
    int rows, classes, features;
    const int* count;  // rows that there are, where that is known on the device alone; or NULL
    const int32_t* labels;
    // statistics of a tile's classes
    Part* parts;  // [rows][tiles.tm]
    float* picked;
    // logits: of all classes (STATS_KEEP), or sums over a part of the features, one matrix after the other (PARTIAL)
    float* z;  // [rows][pitch]
    int k_split;  // features of a part, a multiple of 64
    // gradient of the logits of classes v0 ..
    const Norm* norm;
    bf16_t* dz;  // [rows][pitch]
    int v0, pitch;
    // the mean, left by a work-group behind the tiles of the first piece: losses and labels in the caller's order
    float* loss;  // or NULL
    const float* row_loss;
    const int32_t* all_labels;
    int all_rows;
};

// One tile of the logits: their statistics, the logits or parts of them, or their gradient.
// The classes are the tile's rows m, so that a lane holds four consecutive classes of a row of x and a row's largest logit and sum of
// exponentials take its own values, two exchanges among lanes and one through the LDS; a tile leaves 8 bytes for each of its rows of x.
// Large products are bound by the MFMA under the clock that the power leaves: 3584 counted rows of 2048 features under 65536 classes take
// 745 us, 1.29 PFLOP/s (the same loop fed from the LDS and the L2 with nothing else to do: 1.45); their gradient 1.36 PFLOP/s at
// 7782 x 8192 classes x 4096.  Few rows are bound by the weights' way from memory, on tiles of 64 with four stages in flight: 16 rows
// of 4096 under 131072 classes 171 us, 6.3 TB/s; one row of 1024 under 32768 14 us, 4.8 TB/s.
template <class S, int MODE, bool RAGGED>
__global__ __launch_bounds__(S::THREADS, S::THREADS >= 512 ? 2 : 1) void xent_logits_kernel(const XentArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    if constexpr (MODE == GRAD) {
        if ((int)blockIdx.x == a.tiles.tm * a.tiles.tn) {
            mean_of<S::THREADS>(a.row_loss, a.all_labels, a.all_rows, a.classes, a.loss);
            return;
        }
    }
    int tm, tn;
    tile_of(a.tiles, blockIdx.x, &tm, &tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN, rows = a.count ? *a.count : a.rows;
    if (n0 >= rows) return;
    f32x4 acc[S::FM][S::FN];
    const int k0 = MODE == PARTIAL ? (int)blockIdx.y * a.k_split : 0;
    product<S, RAGGED>(a.w, Operand{a.x.p, a.x.pitch, rows, nullptr, 0}, m0, n0, k0, MODE == PARTIAL ? min(a.features, k0 + a.k_split) : a.features, smem, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave % S::WAVES_M, wn = wave / S::WAVES_M;
    const int mw = m0 + wm * S::WM + (lane >> 4) * 4;  // class of element 0, counted from the piece's first
    const int there = a.classes - a.v0;                // classes from there on
    auto each = [&](int j, auto&& f) __attribute__((always_inline)) {                 // value = f(class offset from mw, value) of the lane's values of one row
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = f(i * 16 + e, acc[i][j][e]);
    };
    if (MODE == PARTIAL || MODE == STATS_KEEP) {
        float* z = a.z + (MODE == PARTIAL ? (size_t)blockIdx.y * a.rows * a.pitch : 0);
        hand_out<S>(acc, smem, [&](int n, int m, f32x4 v) __attribute__((always_inline)) {
            if (n0 + n < rows) *reinterpret_cast<f32x4*>(z + (size_t)(n0 + n) * a.pitch + m0 + m) = v;
        });
        if (MODE == STATS_KEEP) __syncthreads();
    }
    if (MODE == STATS || MODE == STATS_KEEP) {
        Part* meet = reinterpret_cast<Part*>(smem);  // [WAVES_M][BN]
        const bool whole = m0 + S::BM <= there;  // every class of the tile exists
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int col = wn * S::WN + j * 16 + (lane & 15), n = n0 + col;
            const int label = n < rows ? a.labels[n] : -1;
            if (!whole) each(j, [&](int o, float z) { return mw + o < there ? z : -INFINITY; });
            float most = -INFINITY;
            each(j, [&](int, float z) {
                most = fmaxf(most, z);
                return z;
            });
            const float by = most == -INFINITY ? 0.f : most;
            float sum = 0.f;
            each(j, [&](int, float z) {
                sum += exp_of(z - by);  // (of a class that is none, or of -inf: 0)
                return z;
            });
            const int rel = label - mw;
            if (label >= 0 && label < a.classes && rel >= 0 && rel < S::WM && (rel & 15) < 4) {
                float z = 0.f;
                each(j, [&](int o, float v) {
                    z = o == rel ? v : z;
                    return v;
                });
                a.picked[n] = z;
            }
            Part p = {most, sum};
#pragma unroll
            for (int d = 16; d < 64; d <<= 1) p = join(p, {__shfl_xor(p.most, d), __shfl_xor(p.sum, d)});
            if (lane < 16) meet[wm * S::BN + col] = p;
        }
        __syncthreads();
        for (int col = threadIdx.x; col < S::BN; col += S::THREADS) {
            Part p = meet[col];
#pragma unroll
            for (int w = 1; w < S::WAVES_M; ++w) p = join(p, meet[w * S::BN + col]);
            if (n0 + col < rows) a.parts[(size_t)(n0 + col) * a.tiles.tm + tm] = p;
        }
    }
    if (MODE == GRAD) {
        const bool whole = m0 + S::BM <= there;
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int n = n0 + wn * S::WN + j * 16 + (lane & 15);
            const int rel = n < rows ? a.labels[n] - a.v0 - mw : -1;
            const Norm norm = n < rows ? a.norm[n] : Norm{0.f, 0.f};
            each(j, [&](int, float z) { return softmax_of(z, norm); });
            if (rel >= 0 && rel < S::WM && (rel & 15) < 4) each(j, [&](int o, float p) { return o == rel ? p - 1.f : p; });
            if (!whole) each(j, [&](int o, float p) { return mw + o < there ? p : 0.f; });
        }
        hand_out<S>(acc, smem, [&](int n, int m, f32x4 v) __attribute__((always_inline)) {
            // (whole tiles have their place: beyond the last class there are zeros)
            if (n0 + n < rows) *reinterpret_cast<u32x2*>(a.dz + (size_t)(n0 + n) * a.pitch + m0 + m) = pack_bf16x4(v);
        });
    }
}

// What row n's softmax is divided by, and its loss, from the union of its parts.
__device__ __forceinline__ float finish_row(Part p, bool counts, float picked, int n, const int* place, Norm* norm, float* row_loss) {
    const float one = counts ? p.most - picked + logf(p.sum) : 0.f;
    norm[n] = {p.most, log2f(p.sum)};
    row_loss[place ? place[n] : n] = one;
    return one;
}

constexpr int kChunk = 2048;  // classes of a work-group that adds parts of logits up

// Adds the parts of a row's logits up in order; statistics of a chunk of its classes, and (keep) the logits in the first part's place.
// (5 us for 8 parts of 64 rows and 1000 classes, of which a launch is most; the product in one part would leave 240 CUs idle.)
// norm: of rows that are one chunk, which are finished here; or NULL.  place: where row n is in the caller's order (NULL: there).
__global__ __launch_bounds__(256) void xent_join_kernel(float* z, int nparts, int rows, const int* count, int classes, int pitch, const int32_t* labels, bool keep,
                                                        Part* parts, float* picked, Norm* norm, const int* place, float* row_loss) {
    const int n = blockIdx.y, c0 = blockIdx.x * kChunk;
    if (n >= (count ? *count : rows)) return;
    const int label = labels[n];
    const size_t all = (size_t)rows * pitch;
    float* zn = z + (size_t)n * pitch;
    f32x4 v[kChunk / 1024];
    __shared__ float chosen;
    Part p = {-INFINITY, 0.f};
#pragma unroll
    for (int i = 0; i < kChunk / 1024; ++i) {
        const int c = c0 + i * 1024 + threadIdx.x * 4;
        v[i] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (c >= classes) continue;
        f32x4 sum = *reinterpret_cast<const f32x4*>(zn + c);
        for (int s = 1; s < nparts; ++s) {
            const f32x4 t = *reinterpret_cast<const f32x4*>(zn + s * all + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += t[e];
        }
        if (keep) *reinterpret_cast<f32x4*>(zn + c) = sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e < classes) {
                v[i][e] = sum[e];
                p.most = fmaxf(p.most, sum[e]);
                if (c + e == label) picked[n] = chosen = sum[e];
            }
        }
    }
    const float by = p.most == -INFINITY ? 0.f : p.most;
#pragma unroll
    for (int i = 0; i < kChunk / 1024; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p.sum += exp_of(v[i][e] - by);
    __shared__ Part meet[4];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) p = join(p, {__shfl_xor(p.most, d), __shfl_xor(p.sum, d)});
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = p;
    __syncthreads();
    if (threadIdx.x > 0) return;
    p = join(join(meet[0], meet[1]), join(meet[2], meet[3]));
    if (norm) finish_row(p, (unsigned)label < (unsigned)classes, chosen, n, place, norm, row_loss);
    else parts[(size_t)n * gridDim.x + blockIdx.x] = p;
}

// Rows that count, one behind the other: their features (zeros behind the last, up to `to`), labels and places; their number, and the
// factor of the gradient; no loss and no gradient for the others.  A work-group takes `per` rows.
struct GatherArgs {
    const bf16_t* x;
    long pitch;
    const int32_t* labels;
    int rows, features, classes, to, per;
    float scale;
    bf16_t* out;  // [rows][to]
    int32_t* out_labels;
    int *place, *count;
    float *factor, *row_loss;
    bf16_t* dx;  // or NULL
};
__global__ __launch_bounds__(256) void xent_gather_kernel(const GatherArgs a) {
    __shared__ int counts[4];
    const int t = threadIdx.x, lane = t & 63, first = blockIdx.x * a.per;
    auto counted = [&](int n) { return n < a.rows && (unsigned)a.labels[n] < (unsigned)a.classes; };
    int before = 0;
    for (int n = t; n < first; n += 256) before += counted(n) ? 1 : 0;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) before += __shfl_xor(before, d);
    if (lane == 0) counts[t >> 6] = before;
    __syncthreads();
    int at = counts[0] + counts[1] + counts[2] + counts[3];
    const int groups = a.to / 8;
    for (int n = first; n < min(a.rows, first + a.per); ++n) {
        const bf16_t* src = a.x + (long)n * a.pitch;
        if (counted(n)) {
            if (t == 0) {
                a.out_labels[at] = a.labels[n];
                a.place[at] = n;
            }
            for (int g = t; g < groups; g += 256) {
                const int c = g * 8;
                u32x4 v;
                if (c + 8 <= a.features) v = load8_unaligned(src + c);
                else
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int k = c + 2 * h;
                        v[h] = (k < a.features ? (unsigned)src[k] : 0u) | (k + 1 < a.features ? (unsigned)src[k + 1] << 16 : 0u);
                    }
                *reinterpret_cast<u32x4*>(a.out + (size_t)at * a.to + c) = v;
            }
            ++at;
        } else {
            if (t == 0) a.row_loss[n] = 0.f;
            if (a.dx)
                for (int c = t; c < a.features; c += 256) a.dx[(size_t)n * a.features + c] = 0;
        }
    }
    if (t == 0 && first + a.per >= a.rows) {
        *a.count = at;
        *a.factor = at ? a.scale / (float)at : 0.f;
    }
}

// One wavefront a row: what its softmax is divided by, and its loss.  ONE: a single work-group, which leaves the mean as well.
// place: where row n is in the caller's order (NULL: there).
template <bool ONE>
__global__ __launch_bounds__(1024) void xent_rows_kernel(const Part* parts, const float* picked, const int32_t* labels, const int* place, const int* count, int rows,
                                                         int classes, int nparts, Norm* norm, float* row_loss, float* loss) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, there = count ? *count : rows;
    double sum = 0.;
    int counted = 0;
    for (int n = (blockIdx.x * blockDim.x >> 6) + wave; n < there; n += gridDim.x * blockDim.x >> 6) {
        Part p = {-INFINITY, 0.f};
        for (int i0 = 0; i0 < nparts; i0 += 512) {  // eight at a time: their loads do not wait for each other's exponentials
            Part v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * 64 + lane;
                v[u] = i < nparts ? parts[(size_t)n * nparts + i] : Part{-INFINITY, 0.f};
            }
#pragma unroll
            for (int d = 4; d > 0; d >>= 1)
#pragma unroll
                for (int u = 0; u < d; ++u) v[u] = join(v[u], v[u + d]);
            p = join(p, v[0]);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) p = join(p, {__shfl_xor(p.most, d), __shfl_xor(p.sum, d)});
        const bool counts = (unsigned)labels[n] < (unsigned)classes;
        if (lane == 0) {
            sum += finish_row(p, counts, counts ? picked[n] : 0.f, n, place, norm, row_loss);
            counted += counts ? 1 : 0;
        }
    }
    if constexpr (ONE) {
        __shared__ double sums[16];
        __shared__ int counts[16];
        if (lane == 0) {
            sums[wave] = sum;
            counts[wave] = counted;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 16; ++w) {
                sum += sums[w];
                counted += counts[w];
            }
            *loss = counted ? (float)(sum / counted) : 0.f;
        }
    }
}

__global__ __launch_bounds__(1024) void xent_mean_kernel(const float* row_loss, const int32_t* labels, int rows, int classes, float* loss) {
    mean_of<1024>(row_loss, labels, rows, classes, loss);
}

// The gradient of logits that were kept: eight classes a thread, bound by the cache behind the L2s (901 x 30011: 26 us at 6.3 TB/s; computing
// the logits again 84 us).  The work-groups behind the last row: one leaves the mean (labels and losses
// in the caller's order).
__global__ __launch_bounds__(256) void xent_dz_kernel(const float* z, const int* count, int classes, int pitch, const int32_t* labels, const Norm* norms,
                                                      bf16_t* dz, const float* row_loss, const int32_t* all_labels, int rows, float* loss) {
    if ((int)blockIdx.y == rows) {
        if (blockIdx.x == 0) mean_of<256>(row_loss, all_labels, rows, classes, loss);
        return;
    }
    const int n = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (n >= *count || c >= pitch) return;
    const int rel = labels[n] - c;
    const Norm norm = norms[n];
    const size_t at = (size_t)n * pitch + c;
    f32x4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(z + at + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int o = 4 * h + e;
            v[h][e] = c + o < classes ? softmax_of(t[e], norm) - (o == rel ? 1.f : 0.f) : 0.f;
        }
    }
    const u32x2 lo = pack_bf16x4(v[0]), hi = pack_bf16x4(v[1]);
    *reinterpret_cast<u32x4*>(dz + at) = u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// ---- gradients of at most 64 rows: W and dW pass by once, everything else is small ----
constexpr int kFew = 64;

// The gradient of kept logits, transposed: dz[class][64 rows], zeros for rows that do not count or do not exist and for classes behind the
// last.  The work-group behind the last classes leaves the mean and the gradient's factor.
__global__ __launch_bounds__(256) void xent_few_dz_kernel(const float* z, int rows, int classes, int pitch, const int32_t* labels, const Norm* norms, const float* row_loss,
                                                          float scale, bf16_t* dz, float* loss, float* factor) {
    __shared__ __align__(16) bf16_t turn[64 * 72];
    const int t = threadIdx.x;
    if (blockIdx.x == gridDim.x - 1) {
        if (t >= 64) return;
        const bool counts = t < rows && (unsigned)labels[t] < (unsigned)classes;
        const int count = __popcll(__ballot(counts));
        double sum = counts ? row_loss[t] : 0.;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        if (t == 0) {
            *loss = count ? (float)(sum / count) : 0.f;
            *factor = count ? scale / (float)count : 0.f;
        }
        return;
    }
    const int c0 = blockIdx.x * 64, c = (t & 15) * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int n = r * 16 + (t >> 4), label = n < rows ? labels[n] : -1;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if ((unsigned)label < (unsigned)classes) {
            v = *reinterpret_cast<const f32x4*>(z + (size_t)n * pitch + c0 + c);
            const Norm norm = norms[n];
            const int rel = label - c0 - c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = c0 + c + e < classes ? softmax_of(v[e], norm) - (e == rel ? 1.f : 0.f) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) turn[(c + e) * 72 + n] = __builtin_bit_cast(unsigned short, (__bf16)v[e]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int k = r * 32 + (t >> 3), n = (t & 7) * 8;
        *reinterpret_cast<u32x4*>(dz + (size_t)(c0 + k) * 64 + n) = *reinterpret_cast<const u32x4*>(turn + k * 72 + n);
    }
}

// dW of at most 64 rows: a stream of the result.  v_mfma_f32_16x16x32 with the classes as rows; the MFMAs c = 0 .. 7 of a block take the
// features 8 n + c, so that a lane ends with eight consecutive features of four classes and a wavefront stores whole 256-byte
// runs.  The operand of x stays in the registers (rows that do not count as zeros: they may hold anything), a wavefront walks down
// the classes of its 128 features, the wavefronts of a work-group beside each other, so that what is stored at about the same time lies
// together.  Bound by the stores: 8 rows of 2000 features under 56896 classes take 50 us at 4.5 TB/s (66 with a work-group's wavefronts
// under each other), 64 rows of 1024 under 40704 classes 27 us (38 as a product on tiles).
struct FewDwArgs {
    const bf16_t* x;  // [rows][pitch]
    long pitch;
    const bf16_t* dz;  // [classes][64]
    const int32_t* labels;
    const float* factor;
    void* out;  // [classes][features]
    int rows, features, classes, across, per;  // across: wavefronts beside each other; per: blocks of 16 classes of one
    bool f32;
};
template <int STEPS>  // of 32 rows
__device__ __forceinline__ void few_dw(const FewDwArgs& a, int job) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, l4 = lane >> 4;
    const int d0 = job % a.across * 128 + l16 * 8;
    u32x4 x[8][STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        unsigned short h[8][8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int n = s * 32 + l4 * 8 + k;
            u32x4 v = {0u, 0u, 0u, 0u};
            // (the rows are padded to whole groups of eight)
            if (n < a.rows && d0 < a.features && (unsigned)a.labels[n] < (unsigned)a.classes) v = *reinterpret_cast<const u32x4*>(a.x + n * a.pitch + d0);
#pragma unroll
            for (int c = 0; c < 8; ++c) h[k][c] = (unsigned short)(v[c >> 1] >> (16 * (c & 1)));
        }
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w) x[c][s][w] = (unsigned)h[2 * w][c] | ((unsigned)h[2 * w + 1][c] << 16);
    }
    const float factor = *a.factor;
    const int blocks = (a.classes + 15) / 16, first = job / a.across * a.per, last = min(blocks, first + a.per);
    u32x4 next[STEPS];
    auto load = [&](int b) {  // (whole blocks of 64 classes have their place)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) next[s] = *reinterpret_cast<const u32x4*>(a.dz + (size_t)(b * 16 + l16) * 64 + s * 32 + l4 * 8);
    };
    if (first < last) load(first);
    for (int b = first; b < last; ++b) {
        u32x4 g[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) g[s] = next[s];
        if (b + 1 < last) load(b + 1);
        f32x4 acc[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) acc[c] = mfma<false>(g[s], x[c][s], acc[c]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int v = b * 16 + l4 * 4 + e;
            if (v >= a.classes || d0 >= a.features) continue;
            const f32x4 lo = {acc[0][e] * factor, acc[1][e] * factor, acc[2][e] * factor, acc[3][e] * factor};
            const f32x4 hi = {acc[4][e] * factor, acc[5][e] * factor, acc[6][e] * factor, acc[7][e] * factor};
            const size_t at = (size_t)v * a.features + d0;
            if (a.f32) {
                float* p = static_cast<float*>(a.out) + at;
                if (d0 + 8 <= a.features) {
                    __builtin_memcpy(p, &lo, 16);
                    __builtin_memcpy(p + 4, &hi, 16);
                } else {
#pragma unroll
                    for (int c = 0; c < 7; ++c)
                        if (d0 + c < a.features) p[c] = c < 4 ? lo[c & 3] : hi[c & 3];
                }
            } else {
                bf16_t* p = static_cast<bf16_t*>(a.out) + at;
                const u32x2 l = pack_bf16x4(lo), h = pack_bf16x4(hi);
                const u32x4 both = {l[0], l[1], h[0], h[1]};
                if (d0 + 8 <= a.features) {
                    __builtin_memcpy(p, &both, 16);
                } else {
#pragma unroll
                    for (int c = 0; c < 7; ++c)
                        if (d0 + c < a.features) p[c] = (unsigned short)(both[c >> 1] >> (16 * (c & 1)));
                }
            }
        }
    }
}

// Where a gradient goes: out[n][m], bf16 or fp32.  The factor of the mean and of the scale comes in here: dz without it is softmax less one-hot,
// whose label terms lie near -1 and round well; times 1 / rows they would all round by the same share, up to 2^-8 of the
// whole gradient (error of dx and dw at 1001 rows 2.7e-3 so, 2.1e-3 now; 1.7e-3 of it is the rounding of the output).
struct Out {
    void* p;
    int M;
    bool f32;
    const int* place;   // n in the caller's order, or NULL
    const float* factor;
    const int32_t* labels;  // zeros for an n whose label is no class; NULL: there is none such
    int classes;
};
// (what is loaded for a store comes as an argument: behind another store the compiler would load it again)
struct Row {
    int to;
    bool counts;
};
__device__ __forceinline__ Row row_of(const Out& o, int n) { return {o.place ? o.place[n] : n, !o.labels || (unsigned)o.labels[n] < (unsigned)o.classes}; }
__device__ __forceinline__ void put(const Out& o, float factor, Row row, int m, f32x4 v) {
    const size_t at = (size_t)row.to * o.M + m;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = row.counts ? v[e] * factor : 0.f;
    // (rows of any length: the stores need no alignment)
    if (m + 4 <= o.M) {
        if (o.f32) {
            __builtin_memcpy(static_cast<float*>(o.p) + at, &v, 16);
        } else {
            const u32x2 h = pack_bf16x4(v);
            __builtin_memcpy(static_cast<bf16_t*>(o.p) + at, &h, 8);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (m + e >= o.M) continue;
            if (o.f32) static_cast<float*>(o.p)[at + e] = v[e];
            else static_cast<bf16_t*>(o.p)[at + e] = __builtin_bit_cast(unsigned short, (__bf16)v[e]);
        }
    }
}

struct GradArgs {
    Operand a, b;
    Tiles tiles;
    int N, K;
    const int *n_count, *k_count;  // N, K where they are known on the device alone; or NULL
    int k_split;                   // reduction steps of a part, a multiple of 64
    float* part;                   // sums of the parts, [parts][N][M in whole groups of four]; NULL: straight out
    bool first, last;              // of the pieces that add up; of an undivided reduction the last one's sums leave here
    Out out;
};

// out[n][m] = sum over k of a(m, k) * b(n, k): dx with W's features as m, dW with x's.  Neither W nor dz nor x is stored in the order of this
// reduction; the tile transposes them on the way to the MFMA.  Bound as the logits are: dx of 7782 rows, 8192 classes of a piece and 4096
// features 1.27 PFLOP/s with the sums of the pieces before read and written, dW 1.40.
template <class S, bool RAGGED>
__device__ __forceinline__ void grad_tile(const GradArgs& a, int id, int total, unsigned char* smem) {
    // (the tiles of a part of the reduction on as few XCDs as hold them: with every part over all XCDs, dx of 2048 rows, 1024 features and
    // 32768 classes read 671 MB behind the L2s; the whole gradient of 64 x 1024 -> 40704 takes 71 us so, 82 otherwise)
    const int at = of_xcd(id, total), which = at / (a.tiles.tm * a.tiles.tn);
    int tm, tn;
    tile_at(a.tiles, at - which * a.tiles.tm * a.tiles.tn, &tm, &tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN, N = a.n_count ? *a.n_count : a.N, K = a.k_count ? *a.k_count : a.K;
    if (n0 >= N) return;
    const int k0 = which * a.k_split, M = a.out.M, pitch = (M + 3) & ~3;
    f32x4 acc[S::FM][S::FN];
    product<S, RAGGED>(a.a, Operand{a.b.p, a.b.pitch, a.n_count ? N : a.b.extent, nullptr, 0}, m0, n0, k0, min(K, k0 + a.k_split), smem, acc);
    float* part = a.part ? a.part + (size_t)which * a.N * pitch : nullptr;
    const float factor = *a.out.factor;
    struct Old {
        f32x4 sum;
        Row row;
    };
    auto ahead = [&](int n, int m) __attribute__((always_inline)) {
        n = min(n0 + n, N - 1);
        Old old = {{0.f, 0.f, 0.f, 0.f}, {n, true}};
        if (part && !a.first) old.sum = *reinterpret_cast<const f32x4*>(part + (size_t)n * pitch + min(m0 + m, pitch - 4));
        if (a.last) old.row = row_of(a.out, n);
        return old;
    };
    hand_out<S>(acc, smem, ahead, [&](int n, int m, f32x4 v, Old old) __attribute__((always_inline)) {
        n += n0;
        m += m0;
        if (n >= N || m >= M) return;
        if (part) {
            float* p = part + (size_t)n * pitch + m;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += old.sum[e];
            if (!a.last) {
                *reinterpret_cast<f32x4*>(p) = v;
                return;
            }
        }
        put(a.out, factor, old.row, m, v);
    });
}
template <class S, bool RAGGED>
__global__ __launch_bounds__(S::THREADS, S::THREADS >= 512 ? 2 : 1) void xent_grad_kernel(const GradArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    grad_tile<S, RAGGED>(a, blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y, smem);
}

// dx (the first `dx_blocks` work-groups) and dW (the others) of few rows beside each other: the one reads W, the other writes dW, and small ones
// leave most of the chip to each other (64 rows of 4096 under 1000 classes, the whole gradient: 25.5 us, 32.6 with a launch each).
template <class S, bool RAGGED, int STEPS>
__global__ __launch_bounds__(256) void xent_few_grad_kernel(const GradArgs x, const FewDwArgs w, unsigned dx_blocks) {
    extern __shared__ __align__(16) unsigned char smem[];
    if (blockIdx.x < dx_blocks) {
        grad_tile<S, RAGGED>(x, blockIdx.x, dx_blocks, smem);
    } else {
        few_dw<STEPS>(w, (blockIdx.x - dx_blocks) * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
    }
}

// The parts of a divided reduction, added in order, four m a thread: bound by reading them (dx of 2048 x 1024 in eight parts: 13 us, 5.5 TB/s).
__global__ __launch_bounds__(256) void xent_sum_kernel(const float* part, int nparts, int N, const int* count, const Out o) {
    const unsigned per = (unsigned)(o.M + 3) / 4, at = blockIdx.x * 256 + threadIdx.x, n = at / per;
    if ((int)n >= (count ? *count : N)) return;
    const size_t all = (size_t)N * per;
    f32x4 sum = reinterpret_cast<const f32x4*>(part)[at];
    for (int s = 1; s < nparts; ++s) {
        const f32x4 t = reinterpret_cast<const f32x4*>(part)[s * all + at];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += t[e];
    }
    put(o, *o.factor, row_of(o, (int)n), (int)(at - n * per) * 4, sum);
}

// Rows of `len` elements, `pitch` apart, as rows of `to` (a multiple of 8) with zeros behind: one thread for eight elements
// (30011 rows of 1025: 22 us, 5.7 TB/s).
__global__ __launch_bounds__(256) void xent_pad_kernel(const bf16_t* src, long pitch, int len, int to, unsigned groups, unsigned per, bf16_t* dst) {
    for (unsigned g = blockIdx.x * 256 + threadIdx.x; g < groups; g += gridDim.x * 256) {
        const unsigned row = g / per, c = (g - row * per) * 8;
        const bf16_t* s = src + (long)row * pitch;
        u32x4 v;
        if ((int)c + 8 <= len) v = load8_unaligned(s + c);
        else
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int k = (int)c + 2 * h;
                v[h] = (k < len ? (unsigned)s[k] : 0u) | (k + 1 < len ? (unsigned)s[k + 1] << 16 : 0u);
            }
        *reinterpret_cast<u32x4*>(dst + (size_t)row * to + c) = v;
    }
}

// The tiles: k-rows and i-rows of the M and of the N operand.
template <bool M_IROWS, bool N_IROWS>
using Large = Shape<256, 256, 2, 4, 2, M_IROWS, N_IROWS, false>;
template <bool M_IROWS, bool N_IROWS>
using Medium = Shape<128, 128, 2, 2, 4, M_IROWS, N_IROWS, false>;
template <bool M_IROWS, bool N_IROWS>
using Small = Shape<64, 64, 2, 2, 4, M_IROWS, N_IROWS, false>;

template <class S, class Args>
int launch(void (*kernel)(Args), const Args& a, int blocks, unsigned parts, const char* what, hipStream_t st, std::atomic<bool>& allowed) {
    if (!allowed) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) return set_error(WAP_EHIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
        allowed = true;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, parts), dim3(S::THREADS), S::LDS, st, a);
    return check_launch(what);
}
template <class S, int MODE, bool RAGGED>
int launch_logits(XentArgs a, int classes_here, int parts, hipStream_t st) {
    static std::atomic<bool> allowed{false};
    a.tiles = {(classes_here + S::BM - 1) / S::BM, (a.rows + S::BN - 1) / S::BN, 8};
    return launch<S>((void (*)(XentArgs))xent_logits_kernel<S, MODE, RAGGED>, a, a.tiles.tm * a.tiles.tn + (MODE == GRAD && a.loss ? 1 : 0), parts, "xent_logits", st, allowed);
}
template <int MODE, bool RAGGED>
int launch_logits(int tile, const XentArgs& a, int classes_here, int parts, hipStream_t st) {
    return tile == 0 ? launch_logits<Large<false, false>, MODE, RAGGED>(a, classes_here, parts, st)
         : tile == 1 ? launch_logits<Medium<false, false>, MODE, RAGGED>(a, classes_here, parts, st) : launch_logits<Small<false, false>, MODE, RAGGED>(a, classes_here, parts, st);
}
template <int MODE>
int launch_logits(int tile, const XentArgs& a, int classes_here, int parts, hipStream_t st) {
    return a.w.end ? launch_logits<MODE, true>(tile, a, classes_here, parts, st) : launch_logits<MODE, false>(tile, a, classes_here, parts, st);
}
template <bool RAGGED, int STEPS>
int launch_few_grad(GradArgs x, const FewDwArgs& w, int parts, unsigned dw_blocks, hipStream_t st) {
    using S = Small<true, true>;
    static std::atomic<bool> allowed{false};
    const auto kernel = xent_few_grad_kernel<S, RAGGED, STEPS>;
    if (!allowed) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) return set_error(WAP_EHIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
        allowed = true;
    }
    x.tiles = {(x.out.M + S::BM - 1) / S::BM, (x.N + S::BN - 1) / S::BN, 8};
    const unsigned dx_blocks = (unsigned)(parts * x.tiles.tm * x.tiles.tn);
    hipLaunchKernelGGL(kernel, dim3(dx_blocks + dw_blocks), dim3(256), dx_blocks ? S::LDS : 0, st, x, w, dx_blocks);
    return check_launch("xent_few_grad");
}
template <class S, bool RAGGED>
int launch_grad(GradArgs a, int parts, hipStream_t st) {
    static std::atomic<bool> allowed{false};
    a.tiles = {(a.out.M + S::BM - 1) / S::BM, (a.N + S::BN - 1) / S::BN, 8};
    return launch<S>((void (*)(GradArgs))xent_grad_kernel<S, RAGGED>, a, a.tiles.tm * a.tiles.tn, parts, "xent_grad", st, allowed);
}
template <bool N_IROWS, bool RAGGED>
int launch_grad(int tile, const GradArgs& a, int parts, hipStream_t st) {
    return tile == 0 ? launch_grad<Large<true, N_IROWS>, RAGGED>(a, parts, st)
         : tile == 1 ? launch_grad<Medium<true, N_IROWS>, RAGGED>(a, parts, st) : launch_grad<Small<true, N_IROWS>, RAGGED>(a, parts, st);
}
template <bool N_IROWS>
int launch_grad(int tile, const GradArgs& a, int parts, hipStream_t st) {
    if constexpr (!N_IROWS) {  // (dx: the weights may be ragged; rows of x that dW takes have been gathered)
        if (a.a.end) return launch_grad<N_IROWS, true>(tile, a, parts, st);
    }
    return launch_grad<N_IROWS, false>(tile, a, parts, st);
}

int launch_pad(const bf16_t* src, long pitch, int rows, int len, int to, bf16_t* dst, hipStream_t st) {
    const unsigned per = (unsigned)to / 8, groups = (unsigned)rows * per;
    hipLaunchKernelGGL(xent_pad_kernel, dim3(std::min(8192u, (groups + 255) / 256)), dim3(256), 0, st, src, pitch, len, to, groups, per, dst);
    return check_launch("xent_pad");
}

// Tile and division of the reduction of an M x N product: the work on the fullest CU, and what adding the parts up takes.
struct Choice {
    int tile, parts, k_split;
    double us;
};
Choice choose(long M, long N, int K, int most_parts, int largest = 0) {  // largest: of kSides
    static const double beside[4] = {10., 5., 2., 8.};
    const int stages = (K + kStep - 1) / kStep;
    Choice best = {};
    for (int parts = 1; parts <= std::min(most_parts, stages); parts = parts < 4 ? parts + 1 : parts & (parts - 1) ? parts * 4 / 3 : parts * 3 / 2)
        for (int k = largest; k < 3; ++k) {
            const int per = (stages + parts - 1) / parts, there = (stages + per - 1) / per;
            if (there != parts) continue;
            const double count = (double)((M + kSides[k] - 1) / kSides[k]) * ((N + kSides[k] - 1) / kSides[k]) * parts, one = tile_us(k, count, per, beside);
            double us = k == 2 ? std::max(last_small_tile_us(per, count), count * one / kNumCU) : std::ceil(count / kNumCU) * one;
            // a launch, and the parts written and read at 4 TB/s
            if (parts > 1) us += 4. + (double)parts * M * N * 8. / 4e6;
            if (best.parts == 0 || us < best.us) best = {k, parts, per * kStep, us};
        }
    return best;
}

// How a call runs, and where everything lies in its workspace.
struct Layout {
    bool few, gather, pad_x, pad_w, keep;
    int features;        // rounded up to 8 where an operand is copied
    Choice logits;
    int nparts;          // statistics of a row
    int zpitch;          // of kept logits and of parts
    int piece, npieces;  // classes whose gradient exists at a time (a multiple of 256)
    Choice dz, dx, dw;   // (dz: a piece's logits once more)
    size_t norm, picked, factor, count, labels, place, parts, z, dz_at, part, x, w, bytes;
};
size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
constexpr size_t kPieceBytes = (size_t)128 << 20;

Layout layout(const wap_linear_xent_desc& d, bool grads) {
    Layout l = {};
    const size_t N = (size_t)d.rows;
    const bool odd = d.features % 8 != 0;
    l.features = (d.features + 7) & ~7;
    const int all = (d.classes + 255) / 256;
    l.zpitch = all * 256;
    const size_t zbytes = N * (size_t)l.zpitch * 4;
    l.few = grads && d.rows <= kFew && zbytes <= kPieceBytes;
    // Rows that do not count are left out of every product of a gradient (theirs may hold anything: zero times NaN would be NaN), and
    // of a loss alone where the products are worth the copy.
    l.gather = grads ? !l.few : (double)d.rows * d.classes * d.features >= 1e11;
    l.pad_x = !l.gather && (odd || d.x_pitch % 8 != 0);
    // (the tiles take rows of the weights at any 4-byte address, and clear what their last group of 8 holds of the next row)
    l.pad_w = d.features % 2 != 0 || d.w_pitch % 2 != 0;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += up256(bytes);
        return p;
    };
    l.factor = take(4);
    l.count = take(4);
    l.norm = take(N * sizeof(Norm));
    l.picked = take(N * 4);
    if (l.gather) {
        l.labels = take(N * 4);
        l.place = take(N * 4);
    }
    // Logits of all classes that are small enough to lie in the cache are kept for their gradient where computing them again
    // takes longer than writing and reading them.
    // (a row is a step of a grid's second axis there)
    const bool grid = d.rows < 65535;
    l.keep = grads && grid && zbytes <= kPieceBytes;
    l.logits = choose(d.classes, d.rows, l.features, grid ? (int)std::min<size_t>(16, std::max<size_t>(1, kPieceBytes / 2 / zbytes)) : 1);
    l.keep = l.few || (l.keep && (l.logits.parts > 1 || l.logits.us > 4. + (double)N * l.zpitch * 10. / 6e6));
    l.nparts = l.logits.parts > 1 ? (d.classes + kChunk - 1) / kChunk : (d.classes + kSides[l.logits.tile] - 1) / kSides[l.logits.tile];
    l.parts = take(N * (size_t)l.nparts * sizeof(Part));
    if (l.keep || l.logits.parts > 1) l.z = take(zbytes * l.logits.parts);
    if (grads) {
        // pieces of equal size whose gradient of the logits stays in the chip's cache, and its rows within what a tile can address
        const int most = l.few ? all : (int)std::min<size_t>(kMaxPitch / 256, std::max<size_t>(8, kPieceBytes / (512 * N)));
        l.npieces = (all + most - 1) / most;
        const int per = (all + l.npieces - 1) / l.npieces;
        l.piece = per * 256;
        l.npieces = (all + per - 1) / per;
        l.dz_at = take((l.few ? kFew : N) * (size_t)l.piece * 2);
        const int here = std::min(l.piece, d.classes);
        const size_t M4 = (size_t)((d.features + 3) & ~3);
        auto most_parts = [](size_t bytes) { return (int)std::min<size_t>(32, std::max<size_t>(1, kPieceBytes / 2 / bytes)); };
        l.dz = choose(here, d.rows, l.features, 1);
        l.dx = choose(d.features, d.rows, here, most_parts(N * M4 * 4), l.few ? 2 : 0);
        if (!l.few) l.dw = choose(d.features, here, d.rows, most_parts((size_t)here * M4 * 4));
        const size_t xparts = l.npieces > 1 || l.dx.parts > 1 ? l.dx.parts * N * M4 * 4 : 0, wparts = l.dw.parts > 1 ? (size_t)l.dw.parts * here * M4 * 4 : 0;
        // (the sums of dx last from piece to piece, those of dw do not)
        l.part = take(l.npieces > 1 ? xparts + wparts : std::max(xparts, wparts));
    }
    if (l.gather || l.pad_x) l.x = take(N * (size_t)l.features * 2);
    if (l.pad_w) l.w = take((size_t)d.classes * l.features * 2);
    l.bytes = at;
    return l;
}

int validate(const wap_linear_xent_desc* in, wap_linear_xent_desc* d) {
    if (!in) return set_error(WAP_EINVAL, "linear_xent descriptor is NULL");
    *d = *in;
    if (d->rows < 1 || d->features < 1 || d->classes < 1)
        return set_error(WAP_EINVAL, "linear_xent descriptor: every size must be >= 1 (rows=%d features=%d classes=%d)", d->rows, d->features, d->classes);
    if (d->flags & ~WAP_XENT_DW_F32) return set_error(WAP_EINVAL, "linear_xent descriptor: unknown flag bits 0x%x", d->flags);
    if (d->x_pitch == 0) d->x_pitch = d->features;
    if (d->w_pitch == 0) d->w_pitch = d->features;
    if (d->x_pitch < d->features || d->w_pitch < d->features)
        return set_error(WAP_EINVAL, "linear_xent descriptor: a pitch is below the features (x_pitch=%lld w_pitch=%lld features=%d)", (long long)d->x_pitch,
                         (long long)d->w_pitch, d->features);
    if (d->x_pitch > kMaxPitch || d->w_pitch > kMaxPitch) return set_error(WAP_EUNSUPPORTED, "linear_xent descriptor: rows above %ld elements", kMaxPitch);
    if (d->rows > (1 << 24) || d->classes > (1 << 24)) return set_error(WAP_EUNSUPPORTED, "linear_xent descriptor: more than 2^24 rows or classes");
    if ((long long)d->rows * ((d->features + 7) / 8) > 0x7fffffffLL || (long long)d->classes * ((d->features + 7) / 8) > 0x7fffffffLL)
        return set_error(WAP_EUNSUPPORTED, "linear_xent descriptor: an operand has more than 2^34 elements");
    if ((long long)d->rows * d->classes > 1LL << 37)  // (a launch holds less than 2^32 threads)
        return set_error(WAP_EUNSUPPORTED, "linear_xent descriptor: more than 2^37 logits (rows=%d classes=%d)", d->rows, d->classes);
    return WAP_OK;
}

int check(const void* p, const char* name) {
    if (!p) return set_error(WAP_EINVAL, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & 15u) return set_error(WAP_EINVAL, "%s is not 16-byte aligned", name);
    return WAP_OK;
}

struct Call {
    wap_linear_xent_desc d;
    Layout l;
    unsigned char* ws;
    XentArgs a;
};

int statistics(Call& c, const void* x, const void* w, const int32_t* labels, float scale, float* loss, float* row_loss, void* dx, hipStream_t st) {
    const wap_linear_xent_desc& d = c.d;
    const Layout& l = c.l;
    const bf16_t *xp = (const bf16_t*)x, *wp = (const bf16_t*)w;
    long xpitch = d.x_pitch, wpitch = d.w_pitch;
    const bool ragged = !l.pad_w && d.features % 8 != 0;
    int rc;
    XentArgs& a = c.a;
    a = XentArgs{};
    a.labels = labels;
    if (l.gather) {
        GatherArgs g = {};
        g.x = xp; g.pitch = xpitch; g.labels = labels;
        g.rows = d.rows; g.features = d.features; g.classes = d.classes; g.to = l.features;
        g.per = std::max(d.rows < 1024 ? 1 : 4, (d.rows + 2047) / 2048);
        g.scale = scale;
        g.out = (bf16_t*)(c.ws + l.x); g.out_labels = (int32_t*)(c.ws + l.labels);
        g.place = (int*)(c.ws + l.place); g.count = (int*)(c.ws + l.count); g.factor = (float*)(c.ws + l.factor);
        g.row_loss = row_loss; g.dx = (bf16_t*)dx;
        hipLaunchKernelGGL(xent_gather_kernel, dim3((unsigned)(d.rows + g.per - 1) / g.per), dim3(256), 0, st, g);
        if ((rc = check_launch("xent_gather")) != WAP_OK) return rc;
        a.labels = g.out_labels;
        a.count = g.count;
    } else if (l.pad_x) {
        if ((rc = launch_pad(xp, xpitch, d.rows, d.features, l.features, (bf16_t*)(c.ws + l.x), st)) != WAP_OK) return rc;
    }
    if (l.gather || l.pad_x) {
        xp = (const bf16_t*)(c.ws + l.x);
        xpitch = l.features;
    }
    if (l.pad_w) {
        if ((rc = launch_pad(wp, wpitch, d.classes, d.features, l.features, (bf16_t*)(c.ws + l.w), st)) != WAP_OK) return rc;
        wp = (const bf16_t*)(c.ws + l.w);
        wpitch = l.features;
    }
    a.w = {wp, wpitch, d.classes, ragged ? wp + (long)(d.classes - 1) * wpitch + d.features : nullptr, d.features};
    a.x = {xp, xpitch, d.rows, nullptr, 0};
    a.rows = d.rows;
    a.classes = d.classes;
    a.features = l.features;
    a.parts = (Part*)(c.ws + l.parts);
    a.picked = (float*)(c.ws + l.picked);
    a.norm = (const Norm*)(c.ws + l.norm);
    a.z = (float*)(c.ws + l.z);
    a.pitch = l.zpitch;
    a.k_split = l.logits.k_split;
    const int* place = l.gather ? (const int*)(c.ws + l.place) : nullptr;
    const bool mean_later = l.piece > 0;  // the kernel of the gradient leaves it
    if (l.logits.parts > 1) {
        if ((rc = launch_logits<PARTIAL>(l.logits.tile, a, d.classes, l.logits.parts, st)) != WAP_OK) return rc;
        hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)l.nparts, (unsigned)d.rows), dim3(256), 0, st, a.z, l.logits.parts, d.rows, a.count, d.classes, l.zpitch, a.labels,
                           l.keep, a.parts, a.picked, mean_later && l.nparts == 1 ? (Norm*)(c.ws + l.norm) : nullptr, place, row_loss);
        if ((rc = check_launch("xent_join")) != WAP_OK || (mean_later && l.nparts == 1)) return rc;
    } else {
        rc = l.keep ? launch_logits<STATS_KEEP>(l.logits.tile, a, d.classes, 1, st) : launch_logits<STATS>(l.logits.tile, a, d.classes, 1, st);
        if (rc != WAP_OK) return rc;
    }
    if (!mean_later && (d.rows <= 16 || d.rows * (double)l.nparts <= 4096.) && d.rows <= 64) {  // (a wavefront's rows follow one another)
        hipLaunchKernelGGL((xent_rows_kernel<true>), dim3(1), dim3(1024), 0, st, a.parts, a.picked, a.labels, place, a.count, d.rows, d.classes, l.nparts, (Norm*)(c.ws + l.norm),
                           row_loss, loss);
        return check_launch("xent_rows");
    }
    const int waves = d.rows <= 1024 ? 1 : 16;
    hipLaunchKernelGGL((xent_rows_kernel<false>), dim3((unsigned)std::min(4096, (d.rows + waves - 1) / waves)), dim3(64 * waves), 0, st, a.parts, a.picked, a.labels, place, a.count, d.rows,
                       d.classes, l.nparts, (Norm*)(c.ws + l.norm), row_loss, loss);
    if ((rc = check_launch("xent_rows")) != WAP_OK || mean_later) return rc;
    hipLaunchKernelGGL(xent_mean_kernel, dim3(1), dim3(1024), 0, st, row_loss, labels, d.rows, d.classes, loss);
    return check_launch("xent_mean");
}

// one gradient, or a piece's part of it
int launch_sum(const GradArgs& g, const Choice& how, hipStream_t st) {
    const size_t quads = (size_t)g.N * ((g.out.M + 3) / 4);
    hipLaunchKernelGGL(xent_sum_kernel, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, g.part, how.parts, g.N, g.n_count, g.out);
    return check_launch("xent_sum");
}
template <bool N_IROWS>
int gradient(GradArgs g, const Choice& how, hipStream_t st) {
    g.k_split = how.k_split;
    const bool sum = how.parts > 1 && g.last;
    if (how.parts > 1) g.last = false;
    int rc = launch_grad<N_IROWS>(how.tile, g, how.parts, st);
    return rc != WAP_OK || !sum ? rc : launch_sum(g, how, st);
}

int few_gradients(Call& c, const int32_t* labels, float scale, float* loss, const float* row_loss, void* dx, void* dw, hipStream_t st) {
    const wap_linear_xent_desc& d = c.d;
    const Layout& l = c.l;
    const XentArgs& a = c.a;
    bf16_t* dz = (bf16_t*)(c.ws + l.dz_at);
    float* factor = (float*)(c.ws + l.factor);
    hipLaunchKernelGGL(xent_few_dz_kernel, dim3((unsigned)l.piece / 64 + 1), dim3(256), 0, st, a.z, d.rows, d.classes, l.piece, labels, a.norm, row_loss, scale, dz, loss, factor);
    int rc = check_launch("xent_few_dz");
    if (rc != WAP_OK || (!dx && !dw)) return rc;
    GradArgs g = {};
    g.a = {a.w.p, a.w.pitch, d.features, a.w.end, 0};
    g.b = {dz, kFew, kFew, nullptr, 0};
    g.N = d.rows; g.K = d.classes;
    g.part = l.dx.parts > 1 ? (float*)(c.ws + l.part) : nullptr;
    g.k_split = l.dx.k_split;
    g.first = true; g.last = l.dx.parts == 1;
    g.out = {dx, d.features, false, nullptr, factor, labels, d.classes};
    FewDwArgs f = {};
    f.x = a.x.p; f.pitch = a.x.pitch;
    f.dz = dz;
    f.labels = labels;
    f.factor = factor;
    f.out = dw;
    f.rows = d.rows; f.features = d.features; f.classes = d.classes;
    f.f32 = (d.flags & WAP_XENT_DW_F32) != 0;
    // about sixteen wavefronts a CU, each with several blocks of classes for its operand of x
    const int blocks = (d.classes + 15) / 16;
    f.across = (d.features + 127) / 128;
    f.per = std::max(1, std::min(blocks, (int)((long)blocks * f.across / (kNumCU * 16))));
    const unsigned dw_blocks = dw ? (unsigned)(((long)((blocks + f.per - 1) / f.per) * f.across + 3) / 4) : 0;
    const int parts = dx ? l.dx.parts : 0;
    rc = a.w.end ? (d.rows <= 32 ? launch_few_grad<true, 1>(g, f, parts, dw_blocks, st) : launch_few_grad<true, 2>(g, f, parts, dw_blocks, st))
                 : (d.rows <= 32 ? launch_few_grad<false, 1>(g, f, parts, dw_blocks, st) : launch_few_grad<false, 2>(g, f, parts, dw_blocks, st));
    return rc != WAP_OK || parts < 2 ? rc : launch_sum(g, l.dx, st);
}

int gradients(Call& c, const int32_t* labels, float scale, float* loss, const float* row_loss, void* dx, void* dw, hipStream_t st) {
    const wap_linear_xent_desc& d = c.d;
    const Layout& l = c.l;
    XentArgs& a = c.a;
    const Operand w = a.w;
    int rc;
    a.dz = (bf16_t*)(c.ws + l.dz_at);
    a.pitch = l.piece;
    float* part = (float*)(c.ws + l.part);
    const size_t xparts = l.npieces > 1 ? (size_t)l.dx.parts * d.rows * ((d.features + 3) & ~3) : 0;
    for (int p = 0; p < l.npieces; ++p) {
        const int v0 = p * l.piece, here = std::min(l.piece, d.classes - v0);
        a.v0 = v0;
        a.w = {w.p + (long)v0 * w.pitch, w.pitch, here, w.end, w.last_k};
        if (l.keep) {
            hipLaunchKernelGGL(xent_dz_kernel, dim3((unsigned)(l.piece + 2047) / 2048, (unsigned)d.rows + 1), dim3(256), 0, st, a.z, a.count, d.classes, l.piece, a.labels, a.norm, a.dz,
                               row_loss, labels, d.rows, loss);
            rc = check_launch("xent_dz");
        } else {
            a.loss = p == 0 ? loss : nullptr;
            a.row_loss = row_loss;
            a.all_labels = labels;
            a.all_rows = d.rows;
            rc = launch_logits<GRAD>(l.dz.tile, a, here, 1, st);
        }
        if (rc != WAP_OK) return rc;
        if (dx) {
            GradArgs g = {};
            g.a = {a.w.p, w.pitch, d.features, w.end, 0};
            g.b = {a.dz, l.piece, d.rows, nullptr, 0};
            g.N = d.rows; g.K = here;
            g.n_count = a.count;
            g.part = l.npieces > 1 || l.dx.parts > 1 ? part : nullptr;
            g.first = p == 0; g.last = p + 1 == l.npieces;
            g.out = {dx, d.features, false, (const int*)(c.ws + l.place), (const float*)(c.ws + l.factor), nullptr, d.classes};
            if ((rc = gradient<false>(g, l.dx, st)) != WAP_OK) return rc;
        }
        if (dw) {
            GradArgs g = {};
            g.a = {a.x.p, a.x.pitch, d.features, nullptr, 0};
            g.b = {a.dz, l.piece, here, nullptr, 0};
            g.N = here; g.K = d.rows;
            g.k_count = a.count;
            g.part = l.dw.parts > 1 ? part + xparts : nullptr;
            g.first = g.last = true;
            const bool f32 = (d.flags & WAP_XENT_DW_F32) != 0;
            g.out = {(unsigned char*)dw + (size_t)v0 * d.features * (f32 ? 4 : 2), d.features, f32, nullptr, (const float*)(c.ws + l.factor), nullptr, 0};
            if ((rc = gradient<true>(g, l.dw, st)) != WAP_OK) return rc;
        }
    }
    return WAP_OK;
}

}  // namespace

}  // namespace wap

using namespace wap;

#define XENT_TRY(expr)               \
    do {                             \
        const int rc_ = (expr);      \
        if (rc_ != WAP_OK) return rc_; \
    } while (0)

static int begin(const wap_linear_xent_desc* desc, bool grads, const void* x, const void* w, const int32_t* labels, float* loss, float* row_loss, void* ws,
                 size_t ws_bytes, Call* c) {
    XENT_TRY(validate(desc, &c->d));
    XENT_TRY(check(x, "x"));
    XENT_TRY(check(w, "w"));
    XENT_TRY(check(labels, "labels"));
    XENT_TRY(check(loss, "loss"));
    XENT_TRY(check(row_loss, "row_loss"));
    c->l = layout(c->d, grads);
    if (!ws || ws_bytes < c->l.bytes) return set_error(WAP_EWORKSPACE, "linear_xent: workspace of %zu bytes needed, %zu given", c->l.bytes, ws ? ws_bytes : 0);
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return set_error(WAP_EINVAL, "workspace is not 256-byte aligned");
    c->ws = (unsigned char*)ws;
    return WAP_OK;
}

extern "C" {

int wap_linear_xent_workspace_bytes(const wap_linear_xent_desc* desc, int grads, size_t* bytes_out) {
    wap_linear_xent_desc d;
    XENT_TRY(validate(desc, &d));
    if (!bytes_out) return set_error(WAP_EINVAL, "bytes_out is NULL");
    *bytes_out = layout(d, grads != 0).bytes;
    return WAP_OK;
}

int wap_linear_xent_fwd(const wap_linear_xent_desc* desc, const void* x, const void* w, const int32_t* labels, float* loss, float* row_loss, void* ws,
                        size_t ws_bytes, void* stream) {
    Call c;
    XENT_TRY(begin(desc, false, x, w, labels, loss, row_loss, ws, ws_bytes, &c));
    return statistics(c, x, w, labels, 1.f, loss, row_loss, nullptr, (hipStream_t)stream);
}

int wap_linear_xent_grad(const wap_linear_xent_desc* desc, const void* x, const void* w, const int32_t* labels, float scale, float* loss, float* row_loss,
                         void* dx, void* dw, void* ws, size_t ws_bytes, void* stream) {
    Call c;
    XENT_TRY(begin(desc, true, x, w, labels, loss, row_loss, ws, ws_bytes, &c));
    if (!dx && !dw) return set_error(WAP_EINVAL, "linear_xent: dx and dw are both NULL");
    if (dx) XENT_TRY(check(dx, "dx"));
    if (dw) XENT_TRY(check(dw, "dw"));
    if (!std::isfinite(scale)) return set_error(WAP_EINVAL, "linear_xent: scale must be finite");
    XENT_TRY(statistics(c, x, w, labels, scale, loss, row_loss, dx, (hipStream_t)stream));
    return (c.l.few ? few_gradients : gradients)(c, labels, scale, loss, row_loss, dx, dw, (hipStream_t)stream);
}

}  // extern "C"
