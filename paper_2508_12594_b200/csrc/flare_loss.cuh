// Softmax cross entropy of rows projected onto a vocabulary, and its gradients, without the logits.
//
//     l[n, v] = scale x_n . w_v;   lse_n = log sum_v exp l[n, v];   loss_n = lse_n - l[n, label_n]
//     q[n, v] = exp(l[n, v] - lse_n) - [v = label_n];   dX_n = dloss_n scale sum_v q[n, v] w_v;   dW_v = scale sum_n dloss_n q[n, v] x_n
//
// Four matrix products of rows x width x vocabulary (X W^T forward, X W^T again, G^T X and G W backward), of which the logits would be the largest
// matrix by far: 2.1 GB in bfloat16 for 8192 rows and 128256 words, where X and W are 17 and 263 MB.  Forward they stay in tensor memory: a tile's end takes
// them from there to a maximum and a sum of exponentials per row.  Backward they are formed again, a piece of the vocabulary at a time: G, the piece of q in one to
// three values of 16 bits, is written to scratch (bounded), and one launch takes both products from it.  The fourth product is what keeping no logits costs.
//
// Rows without a label are left out, not multiplied by zero: the rows that have one are packed, in their order, before anything else (loss_scan_kernel,
// loss_pack_kernel), their number stays on the device, and all products run over packed rows.  So a padded batch takes the time of its labelled rows, and
// nothing that stands in the others can reach a gradient.  The pass costs two bytes in and out per element of X, and leaves rows that TMA can take whatever stride and alignment X has.
// (Rows of 16 bits that lie well are scored as they stand where they are up to 256, or of any number over up to 2048 words.)
//
// Every product is the same kernel (loss_kernel): pairs of blocks, tiles of 256 x 256 (or 256 x 128), operands by TMA, sums in tensor memory twice over so
// that a tile's end runs under the next tile's products.  It is bound by the tensor pipe.
//
// bfloat16 and float16 are multiplied as they are, G in the same type, rounded once.  bfloat16's G is q where one dloss is that of all rows (next to a label q is next to -1, which is no rounding), else dloss scale q
// (2^-9, as the gradients themselves will be; dloss in a second X instead put the same rounding there, and as many more elements were moved).  float16's G is q times 2^15, so that probabilities down to 2^-29 are
// normal numbers; of a row's own dloss its mantissa is there too (q times 2^14 and up to 2) and its power of two in dX's rows and in a second X, times one more that puts the largest element of that just
// below 2^15: elements of x times dloss are held down to 2^-39 of the largest of them.
// Of a small vocabulary or of few rows G is two values of the type (2^-17, 2^-23), two products of either gradient.
// float32: X, W, G as three bfloat16 values each, which hold all 24 bits over all of float32's range, a product as the six of them that are above 2^-24 of it; sums leave tensor memory, which
// truncates, every 64 of K to be added up in registers.  (Two float16 halves, 22 bits, take three products, but want one power of two for all of X, of W and of a row's dloss: an element
// of 1e9 in one row put the others' losses off by 3e-3, one of 1e13 by 4.)
#pragma once

#include <type_traits>

#include "flare_common.cuh"
#include "flare_ptx.cuh"

namespace flare {

// What the packing leaves for the kernels behind it, on the device.
struct LossInfo {
    uint32_t rows;               // with a label
    float d_scale;               // where dloss is in the second X: that is 1 / d_scale times what it stands for, else 1
};
// Per 1024 rows.
struct LossChunk { uint32_t rows; };

__device__ __forceinline__ int64_t label_at(const void *labels, int wide, long n) {
    return wide ? static_cast<const int64_t *>(labels)[n] : (int64_t) static_cast<const int32_t *>(labels)[n];
}

// A thread's walk over groups of columns of rows, without divisions.
struct LossWalk {
    long row, drow;
    uint32_t group, dgroup, groups;
    __device__ __forceinline__ LossWalk(uint64_t first, uint64_t step, uint32_t groups_) : groups(groups_) {
        row = (long)(first / groups); group = (uint32_t)(first % groups);
        drow = (long)(step / groups); dgroup = (uint32_t)(step % groups);
    }
    __device__ __forceinline__ void next() {
        row += drow; group += dgroup;
        if (group >= groups) { group -= groups; ++row; }
    }
};

constexpr int kLossChunk = 1024, kScanThreads = 256;
struct LossScan {
    const void *labels;
    int wide;
    long rows;
    int V, chunks;
    // blocks beyond the chunks', where there is to be a second X: the largest sum of the binary exponents of an element of x and of its row's dloss (float16)
    int C, x_blocks;
    const void *x;
    long ld_x;
    const float *dloss;
    int *largest;                             // [x_blocks]
    int *rank;                                // [rows]: among the labelled rows of its chunk, or -1
    LossChunk *chunk;
    uint32_t *status;
};
// The binary exponent of v (2^e <= |v| < 2^(e + 1)): -126 for less than a normal number, 0 for what is none.
__device__ __forceinline__ int exponent_of(float v) {
    const int e = (int)(__float_as_uint(v) >> 23 & 255);
    return e == 255 ? 0 : max(e, 1) - 127;
}
constexpr int kNoExponent = -1000;
__device__ __forceinline__ int block_max(int v, int *shared) {
    v = __reduce_max_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < (int)blockDim.x / 32; ++w) v = max(v, shared[w]);
    __syncthreads();
    return v;
}
// Eight columns as they lie in memory; `left` of them are, the others are zeros (vec: all or none).
template <typename T> struct LossEight { uint4 q[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ void eight_of(const T *p, bool vec, int left, LossEight<T> &e) {
    if (vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.q[i] = left > 0 ? reinterpret_cast<const uint4 *>(p)[i] : make_uint4(0, 0, 0, 0);
    } else {
        T *t = reinterpret_cast<T *>(e.q);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) t[i] = p[i];
            else from_f32(t[i], 0.f);
    }
}
__global__ void __launch_bounds__(kScanThreads) loss_scan_kernel(const LossScan a) {
    __shared__ int shared[32];
    __shared__ uint32_t before[33];
    ptx::grid_launch();
    ptx::grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.x == 0 && threadIdx.x < kHeaderBytes / 4) a.status[threadIdx.x] = 0;
    if ((int)blockIdx.x >= a.chunks) {
        const __half *x = static_cast<const __half *>(a.x);
        const bool vec = a.C % 8 == 0 && a.ld_x % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
        constexpr int kBatch = 4;                             // groups of eight columns that are asked for before the first is looked at
        LossWalk walk((uint64_t)(blockIdx.x - a.chunks) * kScanThreads + threadIdx.x, (uint64_t)a.x_blocks * kScanThreads, (uint32_t)(a.C + 7) / 8);
        int most = kNoExponent;
        while (walk.row < a.rows) {
            LossEight<__half> e[kBatch];
            float d[kBatch];                                  // 0: not looked at
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                d[k] = 0.f;
                if (walk.row < a.rows) {
                    const int64_t label = label_at(a.labels, a.wide, walk.row);
                    if (label >= 0 && label < a.V) d[k] = a.dloss[walk.row];
                    if (d[k] != 0.f) eight_of(x + walk.row * a.ld_x + 8 * walk.group, vec, a.C - (int)(8 * walk.group), e[k]);
                }
                walk.next();
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (d[k] == 0.f) continue;
                float v = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = fabsf(__half2float(reinterpret_cast<const __half *>(e[k].q)[i]));
                    if (u <= 65504.f) v = fmaxf(v, u);
                }
                if (v > 0.f) most = max(most, exponent_of(v) + exponent_of(d[k]));
            }
        }
        most = block_max(most, shared);
        if (threadIdx.x == 0) a.largest[blockIdx.x - a.chunks] = most;
        return;
    }
    // four times 256 rows of the chunk, in order
    bool there[kLossChunk / kScanThreads];
#pragma unroll
    for (int k = 0; k < kLossChunk / kScanThreads; ++k) {
        const long n = (long)blockIdx.x * kLossChunk + k * kScanThreads + threadIdx.x;
        there[k] = false;
        if (n < a.rows) {
            const int64_t label = label_at(a.labels, a.wide, n);
            there[k] = label >= 0 && label < a.V;
        }
        const uint32_t m = __ballot_sync(0xffffffffu, there[k]);
        if (lane == 0) before[k * (kScanThreads / 32) + warp] = __popc(m);
    }
    __syncthreads();
    if (warp == 0) {
        const uint32_t own = before[lane];
        uint32_t sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        before[lane] = sum - own;
        if (lane == 31) before[32] = sum;
    }
    __syncthreads();
    if (threadIdx.x == 0) a.chunk[blockIdx.x] = LossChunk{before[32]};
#pragma unroll
    for (int k = 0; k < kLossChunk / kScanThreads; ++k) {
        const long n = (long)blockIdx.x * kLossChunk + k * kScanThreads + threadIdx.x;
        const uint32_t m = __ballot_sync(0xffffffffu, there[k]);
        if (n < a.rows) a.rank[n] = there[k] ? (int)(before[k * (kScanThreads / 32) + warp] + __popc(m & ((1u << lane) - 1))) : -1;
    }
}

struct LossPack {
    const void *labels, *x, *w;
    int wide;
    long rows, cap, ld_x, ld_w, w_rows;       // cap: rows up to whole tiles; w_rows: of W to be packed too (0: it is taken as it stands)
    int C, Cp, V, chunks, pack_blocks, pack_rows;   // Cp: C up to a multiple of eight, above 256 of 64
    const int *rank;                          // the scan's; null: there was none
    const LossChunk *chunk;
    const int *largest;                       // with pd: the scan's
    int x_blocks;
    uint32_t *status;
    LossInfo *info;
    uint16_t *px, *pd, *pw;                   // packed X, packed dloss X (or null), packed W: planes of [cap][Cp], [V][Cp]
    int *index, *label;                       // of packed rows: row, label
    // forward
    float *loss, *lse;                        // 0 where there is no label
    // backward
    const float *lse_in, *dloss;
    float mult;                               // on dloss
    float *lse_of, *gm, *coef;                // of packed rows: lse; what q is multiplied by on its way to G, what dX is multiplied by
    float g_factor;                           // of q in G; 0: all of dloss is there
    void *dx;                                 // rows without a label: zeros
    long ld_dx;
};
constexpr int kPackThreads = 256;             // of a block, which takes 4 to 1024 rows (of one chunk)
// Rows up to which every block finds for itself, in all labels, what the scan would tell it, where there is no second X: a launch less, for a pass over all labels a block.  Forward over 5000 words of 256: 1000 rows
// 14.3 us (with the scan 15.3), 4096 20.7 (21.9), 8192 28.5 (28.7), 16384 47.4 (43.9).
constexpr int kPackAlone = 4096;

// What the products multiply: the type as it is; float32 as three bfloat16 values, each what rounding to those before it has left.
template <typename T> constexpr int kPacked = sizeof(T) == 4 ? 3 : 1;
__device__ __forceinline__ void three_of(float v, uint16_t (&t)[3]) {
    __nv_bfloat16 h = fabsf(v) > 3.3895314e38f ? __float2bfloat16_rz(v) : __float2bfloat16_rn(v);         // (beyond bfloat16's largest: not to infinity)
    t[0] = __bfloat16_as_ushort(h);
    float left = fabsf(v) <= 3.4028234e38f ? v - __bfloat162float(h) : 0.f;
    h = __float2bfloat16_rn(left);
    t[1] = __bfloat16_as_ushort(h);
    t[2] = __bfloat16_as_ushort(__float2bfloat16_rn(left - __bfloat162float(h)));
}
// Eight columns into their planes; those of 16 bits times f, or as they are where not `scaled`.
template <typename T>
__device__ __forceinline__ void pack_eight(const LossEight<T> &e, float f, bool scaled, uint16_t *out, long plane) {
    const T *t = reinterpret_cast<const T *>(e.q);
    __align__(16) uint16_t h[8];
    if constexpr (kPacked<T> == 3) {
        __align__(16) uint16_t m[8], l[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint16_t three[3];
            three_of(to_f32(t[i]), three);
            h[i] = three[0]; m[i] = three[1]; l[i] = three[2];
        }
        *reinterpret_cast<uint4 *>(out + plane) = *reinterpret_cast<const uint4 *>(m);
        *reinterpret_cast<uint4 *>(out + 2 * plane) = *reinterpret_cast<const uint4 *>(l);
    } else {
        if (!scaled) {
            *reinterpret_cast<uint4 *>(out) = e.q[0];
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            T u;
            from_f32(u, to_f32(t[i]) * f);
            h[i] = *reinterpret_cast<const uint16_t *>(&u);
        }
    }
    *reinterpret_cast<uint4 *>(out) = *reinterpret_cast<const uint4 *>(h);
}
template <typename T>
__global__ void __launch_bounds__(kPackThreads) loss_pack_kernel(const LossPack a) {
    __shared__ int shared[32];
    __shared__ uint32_t sums[2][kPackThreads / 32];
    __shared__ int to_row[kLossChunk];                        // of packed X; -1: no label
    __shared__ float d_row[kLossChunk];                       // what x is multiplied by in the second X
    ptx::grid_launch();
    ptx::grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kBatch = 4;                                 // groups of eight columns that are asked for before the first is stored
    const uint32_t groups = (uint32_t)a.Cp / 8;
    if ((int)blockIdx.x >= a.pack_blocks) {                   // W
        const T *w = static_cast<const T *>(a.w);
        const bool vec = a.C % 8 == 0 && a.ld_w * (long)sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(w) & 15) == 0;
        LossWalk walk((uint64_t)(blockIdx.x - a.pack_blocks) * kPackThreads + threadIdx.x, (uint64_t)(gridDim.x - a.pack_blocks) * kPackThreads, groups);
        while (walk.row < a.w_rows) {
            LossEight<T> e[kBatch];
            long at[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                at[k] = walk.row < a.w_rows ? walk.row * a.Cp + walk.group * 8 : -1;
                if (at[k] >= 0) eight_of(w + walk.row * a.ld_w + walk.group * 8, vec, a.C - (int)walk.group * 8, e[k]);
                walk.next();
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (at[k] >= 0) pack_eight<T>(e[k], 1.f, false, a.pw + at[k], a.w_rows * a.Cp);
        }
        return;
    }
    // labelled rows before this block's chunk (alone: before its rows), and in all
    const bool alone = a.rank == nullptr;
    if (alone && blockIdx.x == 0 && threadIdx.x < kHeaderBytes / 4) a.status[threadIdx.x] = 0;
    const long n0 = (long)blockIdx.x * a.pack_rows;
    const int chunk = (int)(n0 / kLossChunk);
    uint32_t base = 0, total = 0;
    if (alone)
        for (long n = threadIdx.x; n < a.rows; n += kPackThreads) {
            const int64_t label = label_at(a.labels, a.wide, n);
            if (label < 0 || label >= a.V) continue;
            ++total;
            if (n < n0) ++base;
        }
    for (int i = alone ? a.chunks : threadIdx.x; i < a.chunks; i += kPackThreads) {
        const LossChunk c = a.chunk[i];
        total += c.rows;
        if (i < chunk) base += c.rows;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        base += __shfl_xor_sync(0xffffffffu, base, o);
        total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    if (lane == 0) { sums[0][warp] = base; sums[1][warp] = total; }
    int d_shift = 0;                                          // binary exponent of d_scale
    if (a.pd) {
        int most = kNoExponent;
        for (int i = threadIdx.x; i < a.x_blocks; i += kPackThreads) most = max(most, a.largest[i]);
        most = block_max(most, shared);
        if (most != kNoExponent) d_shift = min(max(most - 14, -126), 127);
    }
    __syncthreads();
    base = total = 0;
    for (int w = 0; w < kPackThreads / 32; ++w) { base += sums[0][w]; total += sums[1][w]; }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.info = LossInfo{total, ldexpf(1.f, d_shift)};
    const int rows = (int)min((long)a.pack_rows, a.rows - n0);
    if (alone) {                                              // (up to a row a thread)
        __syncthreads();                                      // (sums have been read)
        int64_t label = -1;
        if ((int)threadIdx.x < rows) label = label_at(a.labels, a.wide, n0 + threadIdx.x);
        const bool there = label >= 0 && label < a.V;
        const uint32_t m = __ballot_sync(0xffffffffu, there);
        if (lane == 0) sums[0][warp] = __popc(m);
        __syncthreads();
        int before = 0;
        for (int w = 0; w < warp; ++w) before += (int)sums[0][w];
        to_row[threadIdx.x] = there ? before + __popc(m & ((1u << lane) - 1)) : -1;
    }
    for (int i = threadIdx.x; i < rows; i += kPackThreads) {
        const long n = n0 + i;
        const int rank = alone ? to_row[i] : a.rank[n];
        const long to = rank < 0 ? -1 : (long)base + rank;
        to_row[i] = (int)to;
        if (rank >= 0) {
            a.index[to] = (int)n;
            a.label[to] = (int)label_at(a.labels, a.wide, n);
            if (a.loss == nullptr) {
                const float d = a.dloss ? a.dloss[n] : 1.f;
                const int e = a.dloss ? exponent_of(d) : 0;
                const float two = __uint_as_float((uint32_t)(e + 127) << 23);
                d_row[i] = ldexpf(1.f, min(e - d_shift, 120));            // (beyond 2^38 x is zeros)
                a.lse_of[to] = a.lse_in[n];
                a.gm[to] = a.g_factor == 0.f ? d * a.mult : d / two * a.g_factor;
                a.coef[to] = a.g_factor == 0.f ? 1.f : two * a.mult / a.g_factor;
            }
        } else if (a.loss) {
            a.loss[n] = 0.f;
            a.lse[n] = 0.f;
        }
    }
    __syncthreads();
    const T *x = static_cast<const T *>(a.x);
    T *dx = static_cast<T *>(a.dx);
    const bool vec = a.C % 8 == 0 && a.ld_x * (long)sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    const bool vec_dx = a.C % 8 == 0 && a.ld_dx * (long)sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(dx) & 15) == 0;
    const long plane = a.cap * a.Cp;
    LossWalk walk(threadIdx.x, kPackThreads, groups);
    while (walk.row < rows) {
        LossEight<T> e[kBatch];
        int row[kBatch], col[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            row[k] = (int)walk.row; col[k] = (int)walk.group * 8;
            if (walk.row < rows && to_row[row[k]] >= 0) eight_of(x + (n0 + row[k]) * a.ld_x + col[k], vec, a.C - col[k], e[k]);
            walk.next();
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (row[k] >= rows) break;
            const long to = to_row[row[k]];
            if (to >= 0) {
                pack_eight<T>(e[k], 1.f, false, a.px + to * a.Cp + col[k], plane);
                if (a.pd) pack_eight<T>(e[k], d_row[row[k]], true, a.pd + to * a.Cp + col[k], plane);
            } else if (dx) {
                T *p = dx + (n0 + row[k]) * a.ld_dx + col[k];
                if (col[k] >= a.C) continue;
                if (vec_dx) {
#pragma unroll
                    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = make_uint4(0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (col[k] + i < a.C) from_f32(p[i], 0.f);
                }
            }
        }
    }
    // Backward: zeros up to the next 64 rows, which the products that sum over rows read.  (Others read whole tiles, but a row that is none reaches nothing but its own results,
    // which nobody looks at.)
    if (a.loss == nullptr) {
        const long end = min(a.cap, ((long)max(total, 1u) + 63) / 64 * 64);
        for (long r = total + (long)blockIdx.x * (kPackThreads / 32) + warp; r < end; r += (long)a.pack_blocks * (kPackThreads / 32))
            for (int h = 0; h < kPacked<T>; ++h)
                for (int c = lane * 8; c < a.Cp; c += 256) {
                    *reinterpret_cast<uint4 *>(a.px + h * plane + r * a.Cp + c) = make_uint4(0, 0, 0, 0);
                    if (a.pd) *reinterpret_cast<uint4 *>(a.pd + h * plane + r * a.Cp + c) = make_uint4(0, 0, 0, 0);
                }
    }
}

// ---------------------------------------------------------------- the products
enum { kLossStats = 0, kLossWeights = 1, kLossGrads = 2, kLossTurns = 3 };   // (kLossTurns: kLossStats with tiles by turns)
__host__ __device__ constexpr bool loss_forward(int kind) { return kind == kLossStats || kind == kLossTurns; }
constexpr int kLossThreads = 640, kLossResults = 16;          // warp 0 loads, warp 1 issues, warps 4 to 19 take the sums out of tensor memory
constexpr uint32_t kLossHalfTile = 128 * 128;                 // bytes: 128 rows (or 64 rows of two blocks of columns) of 64 elements
constexpr uint32_t kLossPiece = 2048;                         // a warp's piece of a result on its way out: 32 rows of 64 bytes
// kA, kB: values of 16 bits that an element of a product's two factors is held in; what they come to are the products of the i-th and the j-th of them with i + j below the larger number.
template <int kA, int kB> struct LossShape {
    static constexpr int kStages = 12 / (kA + kB), kProducts = kA > kB ? kA : kB;
    static constexpr uint32_t kStage = (kA + kB) * kLossHalfTile;
};
// 64-deep steps whose sums stay in tensor memory, where every addition truncates: of float32 1 (6 x 4 additions: gradients off by 3.8e-7 to 4.0e-7); of 16-bit factors' logits 8 (a loss over 4096 columns is off by 2e-6 with all of
// them there; the same forward and backward, so that both have the same logits); of the gradients, whose results are rounded to 2^-9 or 2^-12, 64 (of 4 additions, or half as many of 8).
template <int kKind, int kF, int kG> constexpr int kLossDeep = kF == 3 ? 1 : kKind != kLossGrads ? 8 : 64 / kG;
constexpr size_t kLossSmem = 1024 + 6 * 2 * kLossHalfTile + kLossResults * kLossPiece + 256;

struct LossMaps { CUtensorMap x, d, w, g; };                  // in boxes of 64 x 64
struct LossArgs {
    const LossInfo *info;
    uint32_t *status;
    int C, V, bf16;              // bf16: the factors are bfloat16 (else float16)
    long cap;                    // rows up to whole tiles
    float scale;
    int v0, words;               // the piece of the vocabulary: from v0 on
    int width, tiles_v;          // X W^T: columns of a tile, tiles across
    const int *label, *index;
    // X as it stands, all of its rows (up to 256, or over a small vocabulary): labels as they stand, and how many rows
    const void *labels;
    int wide, direct;
    __device__ __forceinline__ int label_of(int row) const {
        if (!direct) return label[row];
        const int64_t l = label_at(labels, wide, row);
        return l >= 0 && l < V ? (int)l : -1;
    }
    uint32_t *gave_up;           // direct: a word for every pair's block, joined behind
    // forward: maximum and sum of tiles_v parts of a row, the label's logit; maxima and logits as they leave the products, before `scale`
    float2 *part;
    float *chosen;
    float *loss, *lse;           // not null: a tile is all of the vocabulary, which finishes its rows
    // backward
    const float *lse_of, *gm, *coef;
    uint16_t *g;                 // planes [cap][ld_g]
    long ld_g;
    int grad_width, tiles_c;     // columns of a gradient's tile, tiles across
    int first, last;             // of the pieces
    void *dw, *dx;
    long ld_dw, ld_dx;
    int dw_vec, dx_vec;          // rows can be written 16 bytes at a time
    float dw_factor;             // scale dloss_scale / g_factor (times d_scale), or 1 where G holds them
    float *acc;                  // dX over the pieces before, by tile: [2 blocks][grad_width columns][128 rows]
    float *slots;                // sums of parts of tiles, likewise, two per pair
};

// Who does what of the two gradients.  Tiles of dW (a piece's words, sums over rows) come first, then tiles of dX (sums over words); whole rounds of
// them are dealt out a tile a pair, so that pairs side by side read the same columns of G at the same time.  Of the rounds that would not be full, either's tiles go to a pair each or are cut along K: the pairs
// that have none whole take equal shares of their steps, and what is less than a tile goes to a slot of the pair's, to be joined.  Which, by the longest pair's steps, where joining counts as 12 (of one gradient)
// or 24 of them: 1999 rows of 200 over 10007 words, 40 tiles of 29 steps and 8 of 157, took 18 us to join with all 48 shared.
// Equal shares begin anywhere along K, so that no two pairs read the same lines of G and W at a time: of a G of half a gigabyte a step then takes half as long again (4096 rows over 64000 words of 1024, the tiles
// of dX shared: 885 us and 4.4 GB read; a pair each, on 64 of 74 pairs: 740 us).  Shares of tiles of few steps
// have many ends (17 rows over 67126 words of 83, forward and backward: 14 tiles of dW for each of three pairs, 156 us; a pair each 84; both with G in one value).
struct LossSplit {
    int tiles_w, tiles_x, deep_w, deep_x, full_w, full_x, pairs;
    int whole_w, whole_x;        // tiles of the last rounds that a pair each takes whole: the first pairs those of dW, the next those of dX
    int sharing;                 // pairs behind them that share the others
    long steps, each;            // of the others; of a pair's, less what is `over`
    int over;
    __device__ __forceinline__ LossSplit(const LossArgs &a, int rows, int pairs_) : pairs(pairs_) {
        const int rb = max(1, (rows + 255) / 256);
        tiles_w = a.dw ? (a.words + 255) / 256 * a.tiles_c : 0;
        tiles_x = a.dx ? rb * a.tiles_c : 0;
        deep_w = max(1, (rows + 63) / 64);
        deep_x = (a.words + 63) / 64;
        // (a round that is nearly full is left as it is)
        auto full = [&](int tiles) { return tiles % pairs * 8 >= 7 * pairs ? tiles : tiles / pairs * pairs; };
        full_w = full(tiles_w);
        full_x = full(tiles_x);
        const int rest_w = tiles_w - full_w, rest_x = tiles_x - full_x;
        const long all_w = (long)rest_w * deep_w, all_x = (long)rest_x * deep_x;
        whole_w = whole_x = 0;
        const float far = 1.f + fminf(0.5f, (float)rows * (float)a.words * 0x1p-29f);
        // how long a share takes: its steps, but four for a tile of fewer (its end runs under the next one's steps).  (Every kernel has to come to the same: nothing here may be fused in one and not in another.)
        auto equal = [&](long steps, int left, int deep) { return __fmul_rn(__fdividef((float)steps, (float)left), far + (deep == 1 ? 3.f : deep == 2 ? 1.f : deep == 3 ? 0.333f : 0.f)); };
        float best = __fadd_rn(equal(all_w + all_x, pairs, rest_w && rest_x ? min(deep_w, deep_x) : rest_w ? deep_w : deep_x), 24.f);
        auto better = [&](int w, int x) {                     // these whole
            const int left = pairs - w - x;
            const long shared = (w ? 0 : all_w) + (x ? 0 : all_x);
            if (left < 0 || (left == 0 && shared > 0)) return;
            const float cost = fmaxf((float)max(w ? deep_w : 0, x ? deep_x : 0), shared > 0 ? __fadd_rn(equal(shared, left, w ? deep_x : deep_w), 12.f) : 0.f);
            if (cost < best) { best = cost; whole_w = w; whole_x = x; }
        };
        better(rest_w, 0);
        better(0, rest_x);
        better(rest_w, rest_x);
        steps = (whole_w ? 0 : all_w) + (whole_x ? 0 : all_x);
        sharing = (int)max(1L, min((long)(pairs - whole_w - whole_x), steps / 4));   // at least four steps a share
        each = steps / sharing;
        over = (int)(steps - each * sharing);
    }
    __device__ __forceinline__ int shared_w() const { return whole_w ? 0 : tiles_w - full_w; }
    __device__ __forceinline__ int shared_x() const { return whole_x ? 0 : tiles_x - full_x; }
    __device__ __forceinline__ long share(int p) const { return p * each + p * over / sharing; }   // (p steps / sharing, without a 64-bit division)
    // The shared tile that step s is of: its first step, depth and number (tiles of dX behind those of dW).
    __device__ __forceinline__ void tile_of(long s, long &start, int &deep, int &tile) const {
        const long w = (long)shared_w() * deep_w;
        if (s < w) {
            const int t = (int)(s / deep_w);
            start = (long)t * deep_w; deep = deep_w; tile = full_w + t;
        } else {
            const int t = (int)((s - w) / deep_x);
            start = w + (long)t * deep_x; deep = deep_x; tile = tiles_w + full_x + t;
        }
    }
};
struct LossUnit { int dx, i, j, kb0, kb1, slot; };            // dx: of that product; tile (i, j); steps; slot: -1: the whole of the tile
// A pair's units of work, one after the other; every role walks through them for itself.
template <int kKind> struct LossUnits;
template <int kKind> struct LossTiles {                       // of X W^T: rows fastest, so that pairs side by side share words
    int i, j, di, dj, rb, tiles_v, deep;
    __device__ __forceinline__ LossTiles(const LossArgs &a, int rows, int pair, int pairs) : rb(max(1, (rows + 255) / 256)), tiles_v(a.tiles_v), deep((a.C + 63) / 64) {
        i = pair % rb; j = pair / rb;
        di = pairs % rb; dj = pairs / rb;
    }
    __device__ __forceinline__ bool next(LossUnit &u) {
        if (j >= tiles_v) return false;
        u = LossUnit{0, i, j, 0, deep, -1};
        i += di; j += dj;
        if (i >= rb) { i -= rb; ++j; }
        return true;
    }
};
template <> struct LossUnits<kLossStats> : LossTiles<kLossStats> { using LossTiles::LossTiles; };
template <> struct LossUnits<kLossTurns> : LossTiles<kLossTurns> { using LossTiles::LossTiles; };
template <> struct LossUnits<kLossWeights> : LossTiles<kLossWeights> { using LossTiles::LossTiles; };
template <> struct LossUnits<kLossGrads> {
    LossSplit s;
    int pair, tiles_c, t, dx;    // next tile of the full rounds, of which gradient (2: none)
    int i, j, i0, j0, di, dj;    // where it is, where the pair's first one is, from one round's to the next's
    bool rest;                   // the pair's whole tile of the last rounds is still to come
    long at, end;
    __device__ __forceinline__ LossUnits(const LossArgs &a, int rows, int pair_, int pairs) : s(a, rows, pairs), pair(pair_), tiles_c(a.tiles_c), t(pair_), dx(0) {
        i = i0 = pair / tiles_c; j = j0 = pair % tiles_c;
        di = pairs / tiles_c; dj = pairs % tiles_c;
        const int me = pair - s.whole_w - s.whole_x;          // among those that share
        rest = me < 0;
        at = end = 0;
        if (me >= 0 && me < s.sharing) { at = s.share(me); end = s.share(me + 1); }
    }
    __device__ __forceinline__ LossUnit whole(int dx, int tile) const { return LossUnit{dx, tile / tiles_c, tile % tiles_c, 0, dx ? s.deep_x : s.deep_w, -1}; }
    __device__ __forceinline__ bool next(LossUnit &u) {
        if (dx == 0 && t >= s.full_w) { dx = 1; t = pair; i = i0; j = j0; }
        if (dx == 1 && t >= s.full_x) dx = 2;
        if (dx < 2) {
            u = LossUnit{dx, i, j, 0, dx ? s.deep_x : s.deep_w, -1};
            t += s.pairs;
            i += di; j += dj;
            if (j >= tiles_c) { j -= tiles_c; ++i; }
            return true;
        }
        if (rest) {
            rest = false;
            u = pair < s.whole_w ? whole(0, s.full_w + pair) : whole(1, s.full_x + pair - s.whole_w);
            return true;
        }
        if (at >= end) return false;
        long start;
        int deep, tile;
        s.tile_of(at, start, deep, tile);
        const bool of_x = tile >= s.tiles_w;
        if (of_x) tile -= s.tiles_w;
        const int kb0 = (int)(at - start), kb1 = (int)min((long)deep, end - start);
        u = LossUnit{of_x, tile / tiles_c, tile % tiles_c, kb0, kb1, kb0 == 0 && kb1 == deep ? -1 : 2 * (pair - s.whole_w - s.whole_x) + (kb0 > 0 ? 0 : 1)};
        at = start + kb1;
        return true;
    }
};

struct LossPipe {
    uint32_t smem0, pieces0, bars, tmem;
    volatile uint32_t *abort_flag;
    uint32_t n, c;               // stages loaded or issued, sets of sums handed over (each role counts for itself)
    int stages;
    __device__ __forceinline__ uint32_t full(uint32_t s) const { return bars + 8 * s; }
    __device__ __forceinline__ uint32_t empty(uint32_t s) const { return bars + 8 * (stages + s); }
    __device__ __forceinline__ uint32_t acc_full(uint32_t b) const { return bars + 8 * (2 * stages + b); }
    __device__ __forceinline__ uint32_t acc_empty(uint32_t b) const { return bars + 8 * (2 * stages + 2 + b); }
};

// The loading warp's part.
template <int kKind, int kA, int kB>
__device__ __forceinline__ void loss_load(LossPipe &q, const LossMaps &m, const LossArgs &a, int rows, int pair, int pairs) {
    using Shape = LossShape<kA, kB>;
    if (!ptx::elect_one()) return;
    const int in_pair = (int)(blockIdx.x & 1);
    asm volatile("fence.proxy.async.global;" ::: "memory");              // (what was stored by the kernels before this, for the loads by TMA)
    LossUnits<kKind> units(a, rows, pair, pairs);
    LossUnit u;
    while (units.next(u)) {
        const int width = kKind == kLossGrads ? a.grad_width : a.width, right = width / 2;
        const int ra = u.i * 256 + in_pair * 128, rb = u.j * width + in_pair * right;
        for (int kb = u.kb0; kb < u.kb1; ++kb, ++q.n) {
            const uint32_t s = q.n % Shape::kStages;
            if (q.n >= Shape::kStages && !ptx::mbar_wait(q.empty(s), (q.n / Shape::kStages - 1) & 1, q.abort_flag, 111)) return;
            const uint32_t at = q.smem0 + s * Shape::kStage, bar = ptx::in_block(q.full(s), 0), bt = at + kA * kLossHalfTile;
            if (in_pair == 0) ptx::mbar_arrive_expect_tx(q.full(s), 2 * (kA * kLossHalfTile + kB * right * 128));
#pragma unroll
            for (int h = 0; h < kA; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t pa = at + h * kLossHalfTile + r * 8192;
                    if (kKind != kLossGrads) ptx::tma_load_3d_for<2>(pa, &m.x, bar, kb * 64, ra + r * 64, h);
                    else if (u.dx) ptx::tma_load_3d_for<2>(pa, &m.g, bar, kb * 64, ra + r * 64, h);
                    else ptx::tma_load_3d_for<2>(pa, &m.g, bar, ra + r * 64, kb * 64, h);
                }
#pragma unroll
            for (int h = 0; h < kB; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t pb = bt + h * kLossHalfTile + r * 8192;
                    if (r * 64 >= right) continue;
                    if (kKind != kLossGrads) ptx::tma_load_3d_for<2>(pb, &m.w, bar, kb * 64, a.v0 + rb + r * 64, h);
                    else if (u.dx) ptx::tma_load_3d_for<2>(pb, &m.w, bar, rb + r * 64, a.v0 + kb * 64, h);
                    else ptx::tma_load_3d_for<2>(pb, &m.d, bar, rb + r * 64, kb * 64, h);
                }
        }
    }
}
// The issuing warp's part (its pair's first block's).
template <int kKind, int kA, int kB, int kDeep>
__device__ __forceinline__ void loss_issue(LossPipe &q, const LossArgs &a, int rows, int pair, int pairs) {
    using Shape = LossShape<kA, kB>;
    if (!ptx::elect_one()) return;
    constexpr uint32_t hi = ptx::desc_hi(1024, 2), value = kLossHalfTile >> 4;
    LossUnits<kKind> units(a, rows, pair, pairs);
    LossUnit u;
    while (units.next(u)) {
        const int width = kKind == kLossGrads ? a.grad_width : a.width;
        const bool a_mn = kKind == kLossGrads && !u.dx, b_mn = kKind == kLossGrads;
        // float32 sums; both factors bfloat16 (1) or float16 (0); which of them lie with K outermost; 256 x width
        const uint32_t idesc = (1u << 4) | ((uint32_t)a.bf16 << 7) | ((uint32_t)a.bf16 << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
                               ((uint32_t)(width >> 3) << 17) | (16u << 24);
        const uint32_t a_lbo = a_mn ? 8192 : 16, b_lbo = b_mn ? 8192 : 16, a_step = (a_mn ? 2048 : 32) >> 4, b_step = (b_mn ? 2048 : 32) >> 4;
        for (int kb = u.kb0; kb < u.kb1; ++q.c) {
            const uint32_t acc = q.tmem + (q.c & 1) * 256;
            if (q.c >= 2 && !ptx::mbar_wait(q.acc_empty(q.c & 1), (q.c / 2 - 1) & 1, q.abort_flag, 112)) return;
            ptx::tc_fence_after();
            for (int k1 = min(kb + kDeep, u.kb1), first = 1; kb < k1; ++kb, ++q.n, first = 0) {
                const uint32_t s = q.n % Shape::kStages;
                if (!ptx::mbar_wait(q.full(s), (q.n / Shape::kStages) & 1, q.abort_flag, 113)) return;
                ptx::tc_fence_after();
                const uint32_t at = q.smem0 + s * Shape::kStage;
                const uint32_t a0 = ptx::desc_lo(at, a_lbo), b0 = ptx::desc_lo(at + kA * kLossHalfTile, b_lbo);
#pragma unroll
                for (int k = 0; k < 4; ++k) {                             // (what lies beyond K is zeros)
                    uint32_t more = !first || k > 0;
#pragma unroll
                    for (int t = Shape::kProducts - 1; t >= 0; --t)       // (small ones first)
#pragma unroll
                        for (int i = 0; i < kA; ++i) {
                            if (t - i < 0 || t - i >= kB) continue;
                            ptx::mma_ss_for<2>(acc, ptx::desc(a0 + k * a_step + i * value, hi), ptx::desc(b0 + k * b_step + (t - i) * value, hi), idesc, more);
                            more = 1;
                        }
                }
                ptx::mma_commit_for<2>(q.empty(s));
            }
            ptx::mma_commit_for<2>(q.acc_full(q.c & 1));
        }
    }
}

// The result warps' parts.  A unit's sums into registers, a row a thread and a quarter of the tile's columns (`cols`, 64 or 32): false if a wait gave up.
template <int kDeep>
__device__ __forceinline__ bool loss_sums(LossPipe &q, int deep, int cols, float (&v)[64]) {
    const int warp = ptx::warp_index(), quad = warp & 3, part = (warp - 4) >> 2;
    const uint32_t acc = q.tmem + ((uint32_t)(quad * 32) << 16) + part * cols;
    for (int kb = 0; kb < deep; kb += kDeep, ++q.c) {
        const bool ok = ptx::mbar_wait(q.acc_full(q.c & 1), (q.c / 2) & 1, q.abort_flag, 114);
        if (!__all_sync(0xffffffffu, ok)) return false;
        ptx::tc_fence_after();
        if (kb == 0) {
#pragma unroll
            for (int k = 0; k < 64; k += 32)
                if (k < cols) ptx::tmem_ld32(acc + (q.c & 1) * 256 + k, reinterpret_cast<uint32_t (&)[32]>(v[k]));
            ptx::tmem_wait_ld();
        } else {
#pragma unroll
            for (int k = 0; k < 64; k += 16) {
                if (k >= cols) break;
                uint32_t u[16];
                ptx::tmem_ld16(acc + (q.c & 1) * 256 + k, u);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) v[k + e] += __uint_as_float(u[e]);
            }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) ptx::mbar_arrive_remote(ptx::in_block(q.acc_empty(q.c & 1), 0));
    }
    return true;
}
// So many result warps at one barrier: whether all of them have their sums, the same in all of their threads.  (A warp whose wait gave up comes here too.)
template <int kBarrier, int kWarps>
__device__ __forceinline__ bool loss_agree(bool ok) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, %3, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all)
                 : "r"((uint32_t)ok), "n"(32 * kWarps), "n"(kBarrier)
                 : "memory");
    return all != 0;
}

// What a result warp needs of its lanes' rows, asked for before it waits for their sums.
struct LossRow { int label, index; float lse, coef; };
template <int kKind>
__device__ __forceinline__ LossRow loss_row(const LossArgs &a, int rows, int row, bool wanted) {
    LossRow r{-1, -1, 0.f, 0.f};
    if (row < rows && wanted) {
        if (kKind != kLossGrads) r.label = a.label_of(row);
        if (kKind == kLossWeights) r.lse = a.lse_of[row];
        if (kKind == kLossGrads || (loss_forward(kKind) && a.loss)) r.index = a.index[row];
        if (!loss_forward(kKind)) r.coef = kKind == kLossWeights ? a.gm[row] : a.coef[row];
    }
    return r;
}

// Exponentials are taken of differences of logits, each rounded once: with a fused multiply-add to a rounded maximum a row whose logits reach 1e8 would have e^4 in the place of 1.  So statistics are of
// sums as they leave the products, in units of which c2 = scale / ln 2 makes exponents, and a logit is rounded (times scale) before lse goes off it.
constexpr float kLossLog2e = 1.4426950408889634f;
__device__ __forceinline__ float loss_from(float m) { return m == -INFINITY ? 0.f : m; }
// Forward: maximum and sum of exponentials of a row's `left` (up to 64) columns.
struct LossStat { float m, l; };
__device__ __forceinline__ LossStat loss_stat(float (&v)[64], int left, float c2) {
    if (left < 64) {
#pragma unroll
        for (int e = 0; e < 64; ++e) v[e] = e < left ? v[e] : -INFINITY;
    }
    float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int e = 4; e < 60; e += 8)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[i] = ptx::max3(mx[i], v[e + i], v[e + 4 + i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) mx[i] = fmaxf(mx[i], v[60 + i]);
    const float m = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), ref = loss_from(m);
    float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int e = 0; e < 64; e += 2) {
        const float2 x = __fmul2_rn(__fadd2_rn(make_float2(v[e], v[e + 1]), make_float2(-ref, -ref)), make_float2(c2, c2));
        l[e >> 1 & 1] = __fadd2_rn(l[e >> 1 & 1], make_float2(ptx::ex2(x.x), ptx::ex2(x.y)));
    }
    return LossStat{m, (l[0].x + l[0].y) + (l[1].x + l[1].y)};
}
// The two sides of a sum of exponentials as one.
__device__ __forceinline__ LossStat loss_both(LossStat a, LossStat b, float c2) {
    const float m = fmaxf(a.m, b.m), ref = loss_from(m);
    return LossStat{m, a.l * ptx::ex2((a.m - ref) * c2) + b.l * ptx::ex2((b.m - ref) * c2)};
}
template <int N> __device__ __forceinline__ LossStat loss_all(const LossStat (&s)[N], float c2) {
    float m = s[0].m;
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, s[i].m);
    const float ref = loss_from(m);
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) l += s[i].l * ptx::ex2((s[i].m - ref) * c2);
    return LossStat{m, l};
}
// lse, rounded as the backward takes a logit off it: where one word is all there is both are the same number.  And a row's loss, of which nothing but log l is left where the label is the maximum.
__device__ __forceinline__ float loss_lse(LossStat s, float scale) { return __fadd_rn(__fmul_rn(s.m, scale), logf(s.l)); }
__device__ __forceinline__ float loss_of(LossStat s, float chosen, float scale) { return (s.m - chosen) * scale + logf(s.l); }
// The value at place `at` (0 to 63), by halves of sixteen at a time.
__device__ __forceinline__ float loss_pick(const float (&v)[64], int at) {
    float r = 0.f;
#pragma unroll
    for (int k = 0; k < 64; k += 16) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = at & 8 ? v[k + e + 8] : v[k + e];
#pragma unroll
        for (int n = 4; n > 0; n >>= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) t[e] = at & n ? t[e + n] : t[e];
        r = at >> 4 == k / 16 ? t[0] : r;
    }
    return r;
}
// What four (or two) warps' columns of a tile say of their rows, joined in shared memory; `joint`: [warps - 1][128 rows], then the labels' logits.
__device__ __forceinline__ void loss_row_out(const LossArgs &a, const LossRow &r, int j, int row, int rows, LossStat s, const float *chosen, float scale) {
    if (row >= rows) return;
    if (a.loss) {
        a.loss[r.index] = loss_of(s, *chosen, scale);
        a.lse[r.index] = loss_lse(s, scale);
    } else {
        a.part[(long)j * a.cap + row] = make_float2(s.m, s.l);
    }
}
__device__ __forceinline__ LossStat loss_columns(const LossArgs &a, float (&v)[64], int at, int cols, int left, int row, float c2, float *chosen) {
    const bool mine = at >= 0 && at < cols;
    if (__any_sync(0xffffffffu, mine)) {
        const float c = loss_pick(v, at);
        if (mine) *(a.loss ? chosen : a.chosen + row) = c;
    }
    return left > 0 ? loss_stat(v, min(cols, left), c2) : LossStat{-INFINITY, 0.f};
}
constexpr int kJoint = 4 * 128;                               // float2 of a place; places are written in turn: one again behind the next tile's barrier
// A tile by all sixteen warps, a quarter of the columns each.
template <int kF>
__device__ __forceinline__ bool loss_stats(LossPipe &q, const LossArgs &a, const LossUnit &u, const LossRow &r, float scale, int rows, int row, int cols, float2 *joint) {
    const float c2 = scale * kLossLog2e;
    const int warp = ptx::warp_index(), part = (warp - 4) >> 2, local = (warp & 3) * 32 + (threadIdx.x & 31), col0 = u.j * a.width + part * cols;
    float *chosen = reinterpret_cast<float *>(joint + 3 * 128) + local;
    float v[64];
    const bool ok = loss_sums<kLossDeep<kLossStats, kF, 1>>(q, u.kb1, cols, v);
    LossStat s[4] = {{-INFINITY, 0.f}, {-INFINITY, 0.f}, {-INFINITY, 0.f}, {-INFINITY, 0.f}};
    if (ok && row - local % 32 < rows) s[0] = loss_columns(a, v, r.label - col0, cols, a.V - col0, row, c2, chosen);   // (some of the warp's rows are rows)
    if (part > 0) joint[(part - 1) * 128 + local] = make_float2(s[0].m, s[0].l);
    if (!loss_agree<1, kLossResults>(ok)) return false;
    if (part == 0) {
#pragma unroll
        for (int p = 0; p < 3; ++p) s[p + 1] = LossStat{joint[p * 128 + local].x, joint[p * 128 + local].y};
        loss_row_out(a, r, u.j, row, rows, loss_all(s, c2), chosen, scale);
    }
    return true;
}
// Tiles in turn by two sets of eight warps, half of the columns each in two steps, where one set of sums is all there is (up to 512 columns of 16 bits): then the sums come quicker than a tile's end, and with all warps
// at the same tile, which wait for one another, the special-function units rest while the others' maxima, labels and joins are formed (forward of 131072 rows of 128 over 256 words: 27.4 us then, 22.9 in turns; of 37137 over 25943: 409 and 334).
__device__ __forceinline__ bool loss_stats_by_turns(LossPipe &q, const LossArgs &a, const LossUnit &u, const LossRow &r, float scale, int rows, int row, float2 *joint) {
    const float c2 = scale * kLossLog2e;
    const int warp = ptx::warp_index(), part = (warp - 4) >> 2, set = part >> 1, half = part & 1, local = (warp & 3) * 32 + (threadIdx.x & 31), cols = a.width / 2;
    const uint32_t acc = q.tmem + ((uint32_t)((warp & 3) * 32) << 16) + half * cols + (q.c & 1) * 256;
    float *chosen = reinterpret_cast<float *>(joint + 3 * 128) + local;
    bool ok = ptx::mbar_wait(q.acc_full(q.c & 1), (q.c / 2) & 1, q.abort_flag, 114);
    ok = __all_sync(0xffffffffu, ok);
    LossStat s[2] = {{-INFINITY, 0.f}, {-INFINITY, 0.f}};
    const int col0 = u.j * a.width + half * cols;
    if (ok) {
        ptx::tc_fence_after();
#pragma unroll 1
        for (int k = 0; 64 * k < cols; ++k) {
            float v[64];
            ptx::tmem_ld32(acc + 64 * k, reinterpret_cast<uint32_t (&)[32]>(v[0]));
            ptx::tmem_ld32(acc + 64 * k + 32, reinterpret_cast<uint32_t (&)[32]>(v[32]));
            ptx::tmem_wait_ld();
            if (64 * (k + 1) >= cols) {
                ptx::tc_fence_before();
                __syncwarp();
                if ((threadIdx.x & 31) == 0) ptx::mbar_arrive_remote(ptx::in_block(q.acc_empty(q.c & 1), 0));
            }
            if (row - local % 32 < rows) {
                s[1] = loss_columns(a, v, r.label - col0 - 64 * k, 64, a.V - col0 - 64 * k, row, c2, chosen);
                s[0] = loss_all(s, c2);
            }
        }
    }
    if (half > 0) joint[local] = make_float2(s[0].m, s[0].l);
    if (!(set ? loss_agree<2, kLossResults / 2>(ok) : loss_agree<1, kLossResults / 2>(ok))) return false;
    if (half == 0) {
        s[1] = LossStat{joint[local].x, joint[local].y};
        loss_row_out(a, r, u.j, row, rows, loss_all(s, c2), chosen, scale);
    }
    return true;
}

// Where 16 bytes of a row of 64 lie in a piece: neither rows a lane nor four lanes a row meet a bank conflict.
__device__ __forceinline__ uint32_t piece_at(int row, int chunk) { return row * 64 + ((chunk ^ (row >> 1 & 3)) << 4); }
// Backward: q of 32 rows and 32 columns at a time, as kG values of 16 bits, to G by way of shared memory, so that four lanes write 64 bytes of a row.
template <int kG>
__device__ __forceinline__ void loss_weights(uint32_t piece, const LossArgs &a, const LossRow &r, float scale, int rows, int row, int local0, int cols, float (&v)[64]) {
    const int lane = threadIdx.x & 31, col0 = a.v0 + local0;
    const bool in = row < rows;
    const int at = r.label - col0;                                       // (no label: below zero)
    const float lse = r.lse, f = r.coef;
    const int words = in ? a.V - col0 : 0;
    // the label's, where it is among the columns: put into the piece on its own (p - 1 in one function: of a row that has learned its label ex2's error would be most of it)
    const bool mine = at >= 0 && at < cols;
    float own = 0.f;
    if (__any_sync(0xffffffffu, mine)) own = expm1f(__fsub_rn(__fmul_rn(loss_pick(v, at), scale), lse)) * f;
#pragma unroll
    for (int k = 0; k < 64; k += 32) {
        if (k >= cols) break;
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            // (products one by one: two at a time came out fused with the addition, whatever their rounding said)
            const float2 d = __fadd2_rn(make_float2(__fmul_rn(v[k + e], scale), __fmul_rn(v[k + e + 1], scale)), make_float2(-lse, -lse)), x = __fmul2_rn(d, make_float2(kLossLog2e, kLossLog2e));
            const float2 y = __fmul2_rn(make_float2(ptx::ex2(x.x), ptx::ex2(x.y)), make_float2(f, f));
            v[k + e] = y.x;
            v[k + e + 1] = y.y;
        }
        if (words - k < 32) {                                            // beyond the vocabulary, or rows that are none: zeros whatever the sums hold
#pragma unroll
            for (int e = 0; e < 32; ++e)
                if (e >= words - k) v[k + e] = 0.f;
        }
#pragma unroll
        for (int h = 0; h < kG; ++h) {
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float &x = v[k + 8 * e + 2 * i], &y = v[k + 8 * e + 2 * i + 1];
                    if (kG == 3 || a.bf16) {
                        w[i] = ptx::pack_bf16(x, y);
                        if (h + 1 < kG) {                                 // (what is left is the next one's)
                            x -= __uint_as_float(w[i] << 16);
                            y -= __uint_as_float(w[i] & 0xffff0000u);
                        }
                    } else {
                        const __half2 t = __floats2half2_rn(x, y);
                        w[i] = *reinterpret_cast<const uint32_t *>(&t);
                        if (h + 1 < kG) {
                            const float2 b = __half22float2(t);
                            x -= b.x;
                            y -= b.y;
                        }
                    }
                }
                ptx::sts128(piece + piece_at(lane, e), w);
            }
            if (mine && (at & ~31) == k) {
                uint16_t bits;
                if (kG == 3 || a.bf16) {
                    const __nv_bfloat16 t = __float2bfloat16_rn(own);
                    bits = __bfloat16_as_ushort(t);
                    own -= __bfloat162float(t);
                } else {
                    const __half t = __float2half_rn(own);
                    bits = __half_as_ushort(t);
                    own -= __half2float(t);
                }
                asm volatile("st.shared.b16 [%0], %1;" ::"r"(piece + piece_at(lane, at >> 3 & 3) + (at & 7) * 2), "h"(bits) : "memory");
            }
            __syncwarp();
            uint16_t *out = a.g + ((long)h * a.cap + (row - lane) + (lane >> 2)) * a.ld_g + local0 + k + (lane & 3) * 8;
#pragma unroll
            for (int e = 0; e < 4; ++e) *reinterpret_cast<float4 *>(out + (long)8 * e * a.ld_g) = ptx::lds128(piece + piece_at(8 * e + (lane >> 2), lane & 3));
        }
    }
}

// 32 rows (a row a lane, to go to row `to` of the output; -1: nowhere) of 32 columns from c0 on, times f, by way of shared memory: rows on 16-byte boundaries by four lanes, 64 bytes a row and instruction (32 took
// twice the time, which bounds gradients with few steps a tile: 18935 rows of 1536 over six words, G in one value); others by lanes with neighbouring columns, a row at a time, eight rows' loads before their stores (3159 rows of 2373 over 23 words,
// G in one value, forward and backward: 162 us one by one, 93 so).
template <typename E>
__device__ __forceinline__ void loss_out(uint32_t piece, E *out, long ld, int vec, int to, int c0, int C, float f, const float *v) {
    const int lane = threadIdx.x & 31;
    constexpr int kStep = 64 / (int)sizeof(E), kLane = 16 / (int)sizeof(E);      // columns of a piece, of 16 bytes
#pragma unroll
    for (int k = 0; k < 32; k += kStep) {
        __syncwarp();
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            __align__(16) E e[kLane];
#pragma unroll
            for (int i = 0; i < kLane; ++i) from_f32(e[i], v[k + kLane * g + i] * f);
            ptx::sts128(piece + piece_at(lane, g), reinterpret_cast<const uint32_t *>(e));
        }
        __syncwarp();
        if (vec) {
            const int c = c0 + k + kLane * (lane & 3);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 8 * e + (lane >> 2), t = __shfl_sync(0xffffffffu, to, r);
                const float4 x = ptx::lds128(piece + piece_at(r, lane & 3));
                if (t >= 0 && c < C) *reinterpret_cast<float4 *>(out + (long)t * ld + c) = x;
            }
        } else {
            using Word = typename std::conditional<sizeof(E) == 4, uint32_t, uint16_t>::type;
            const int col = lane % kStep, c = c0 + k + col;
            const uint32_t from = (col % kLane) * (uint32_t)sizeof(E);
            // (eight loads before their stores: each on its own is a wait for shared memory)
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 8 * (32 / kStep)) {
                Word x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t at = piece + piece_at(r0 + i * (32 / kStep) + lane / kStep, col / kLane) + from;
                    if constexpr (sizeof(E) == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x[i]) : "r"(at) : "memory");
                    else asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x[i]) : "r"(at) : "memory");
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = __shfl_sync(0xffffffffu, to, r0 + i * (32 / kStep) + lane / kStep);
                    if (t >= 0 && c < C) reinterpret_cast<Word *>(out)[(long)t * ld + c] = x[i];
                }
            }
        }
    }
}
// 32 columns of a gradient's tile that are complete, tile-local from col on.
template <typename E>
__device__ __forceinline__ void loss_gradient(uint32_t piece, const LossArgs &a, const LossInfo &info, const LossRow &r, int dx, int i, int j, int block, int quad, int col, float *v) {
    const int lane = threadIdx.x & 31, local = i * 256 + block * 128 + quad * 32 + lane, c0 = j * a.grad_width + col;
    if (c0 >= a.C) return;
    if (!dx) {
        const float f = a.dw_factor * info.d_scale;
        loss_out<E>(piece, static_cast<E *>(a.dw), a.ld_dw, a.dw_vec, local < a.words ? a.v0 + local : -1, c0, a.C, f, v);
        return;
    }
    if (!a.first || !a.last) {
        float *acc = a.acc + ((((long)i * a.tiles_c + j) * 2 + block) * a.grad_width + col) * 128 + quad * 32 + lane;
        if (!a.first) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] += acc[e * 128];
        }
        if (!a.last) {
#pragma unroll
            for (int e = 0; e < 32; ++e) acc[e * 128] = v[e];
            return;
        }
    }
    const float f = r.coef;
    loss_out<E>(piece, static_cast<E *>(a.dx), a.ld_dx, a.dx_vec, r.index, c0, a.C, f, v);
}

// kF: values of 16 bits to an element of X and W; kG: to one of G.
template <int kKind, int kF, int kG, typename E>
__global__ void __launch_bounds__(kLossThreads, 1) loss_kernel(const __grid_constant__ LossMaps maps, const LossArgs a) {
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag;
    constexpr int kA = kKind == kLossGrads ? kG : kF, kDeep = kLossDeep<kKind, kF, kG>;
    using Shape = LossShape<kA, kF>;
    LossPipe q;
    q.smem0 = ptx::smem_u32(ptx::align_1024(raw));
    q.pieces0 = q.smem0 + Shape::kStages * Shape::kStage;
    q.bars = q.pieces0 + kLossResults * kLossPiece;
    q.abort_flag = &abort_flag;
    q.n = q.c = 0;
    q.stages = Shape::kStages;
    constexpr bool by_turns = kKind == kLossTurns;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int s = 0; s < Shape::kStages; ++s) { ptx::mbar_init(q.full(s), 1); ptx::mbar_init(q.empty(s), 1); }
        for (int b = 0; b < 2; ++b) { ptx::mbar_init(q.acc_full(b), 1); ptx::mbar_init(q.acc_empty(b), by_turns ? kLossResults : 2 * kLossResults); }
        ptx::fence_mbar_init();
    }
    if (ptx::warp_index() == 1) ptx::tmem_alloc_for<2>(ptx::smem_u32(&tmem_slot), 512);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_meet();
    ptx::tc_fence_after();
    q.tmem = tmem_slot;
    ptx::grid_launch();
    ptx::grid_wait();
    const int warp = ptx::warp_index(), pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1), in_pair = (int)(blockIdx.x & 1);
    const LossInfo info = loss_forward(kKind) && a.direct ? LossInfo{(uint32_t)a.direct, 1.f} : *a.info;
    const int rows = (int)info.rows;
    // Registers of the launch, 640 x 96 (every form's: the split counts on it), as 128 x 40 (the loading and the issuing warp, two that idle) and 512 x 104.  Sixteen result warps with a quarter of the columns each: with eight and half of them, which
    // had 168, their own chain of waits took as long as four products (37137 rows of 128 over 25943 words: 469 us).
    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        loss_load<kKind, kA, kF>(q, maps, a, rows, pair, pairs);
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (in_pair == 0) loss_issue<kKind, kA, kF, kDeep>(q, a, rows, pair, pairs);
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int quad = warp & 3, part = (warp - 4) >> 2, lane = threadIdx.x & 31;
        const int cols = (kKind == kLossGrads ? a.grad_width : a.width) / 4;
        const uint32_t piece = q.pieces0 + (warp - 4) * kLossPiece;
        auto row_of = [&](const LossUnit &u) { return u.i * 256 + in_pair * 128 + quad * 32 + lane; };
        LossUnits<kKind> units(a, rows, pair, pairs);
        LossUnit u, next;
        float2 *joint = reinterpret_cast<float2 *>(ptx::align_1024(raw) + Shape::kStages * Shape::kStage);
        bool more = units.next(u);
        if (by_turns && part >= 2) { more = units.next(u); q.c = 1; }     // (the second set begins with the second tile)
        LossRow r = loss_row<kKind>(a, rows, row_of(u), more && (kKind != kLossGrads || u.dx)), r_next;
        for (uint32_t turn = 0; more; u = next, r = r_next, ++turn) {
            more = units.next(next);                          // (its rows are asked for a unit ahead)
            if (by_turns && more) more = units.next(next);
            r_next = loss_row<kKind>(a, rows, row_of(next), more && (kKind != kLossGrads || next.dx));
            const int row = row_of(u);
            if constexpr (kKind == kLossStats) {
                if (!loss_stats<kF>(q, a, u, r, a.scale, rows, row, cols, joint + (turn & 1) * kJoint)) break;
            } else if constexpr (kKind == kLossTurns) {
                if (!loss_stats_by_turns(q, a, u, r, a.scale, rows, row, joint + (2 * (part >> 1) + (turn & 1)) * kJoint)) break;
                q.c += 2;
            } else {
                float v[64];
                if (!loss_sums<kDeep>(q, u.kb1 - u.kb0, cols, v)) break;
                if constexpr (kKind == kLossWeights) loss_weights<kG>(piece, a, r, a.scale, rows, row, u.j * a.width + part * cols, cols, v);
                else if (u.slot >= 0) {
                    float *slot = a.slots + (((long)u.slot * 2 + in_pair) * a.grad_width + part * cols) * 128 + quad * 32 + lane;
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (e < cols) slot[e * 128] = v[e];
                } else {
#pragma unroll
                    for (int k = 0; k < 64; k += 32)
                        if (k < cols) loss_gradient<E>(piece, a, info, r, u.dx, u.i, u.j, in_pair, quad, part * cols + k, v + k);
                }
            }
        }
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    let_arrive(q.abort_flag);
    ptx::cluster_meet();                                      // (nobody's shared or tensor memory is needed any more)
    if (threadIdx.x == 0) {
        if (loss_forward(kKind) && a.direct) a.gave_up[blockIdx.x] = abort_flag;
        else if (abort_flag != 0) *a.status = abort_flag;
    }
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_for<2>(q.tmem, 512);
    }
}

// Tiles whose K several pairs have shared: 32 rows and 32 columns by one warp, or, where many pairs have (a few tiles summed over many rows), by 2, 4 or 8 that take their
// shares in turn and are added up in order.
constexpr int kJoinWarps = 8, kJoinCols = 32;
template <typename E>
__global__ void __launch_bounds__(32 * kJoinWarps, 2) loss_join_kernel(const LossArgs a, int pairs) {
    __shared__ __align__(128) uint8_t pieces[kJoinWarps][4096];
    ptx::grid_launch();
    ptx::grid_wait();
    const LossInfo info = *a.info;
    const LossSplit s(a, (int)info.rows, pairs);
    if (s.steps == 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks_of_tile = 8 * (a.grad_width / kJoinCols);   // (2 blocks, 4 quarters of rows)
    const int rest_w = s.shared_w(), rest_all = rest_w + s.shared_x();
    const long shares = max(s.deep_w, s.deep_x) / max(1L, s.each);                                // of a tile, about
    const int team = shares < 4 ? 1 : shares < 8 ? 2 : shares < 16 ? 4 : 8, member = warp % team;
    const long items = (long)rest_all * blocks_of_tile, step = (long)gridDim.x * (kJoinWarps / team);
    for (long first = (long)blockIdx.x * (kJoinWarps / team); first < items; first += step) {               // (the same for all warps of the block)
        const long at = first + warp / team;
        const int rest = (int)at / blocks_of_tile, part = (int)at - rest * blocks_of_tile, block = part & 1, quad = part >> 1 & 3, col = (part >> 3) * kJoinCols;
        const bool dx = rest >= rest_w;
        const long start = dx ? (long)rest_w * s.deep_w + (long)(rest - rest_w) * s.deep_x : (long)rest * s.deep_w, end = start + (dx ? s.deep_x : s.deep_w);
        const int tile = dx ? s.full_x + rest - rest_w : s.full_w + rest;
        float v[kJoinCols];
#pragma unroll
        for (int e = 0; e < kJoinCols; ++e) v[e] = 0.f;
        bool shared = false;
        if (at < items) {
            // the first pair whose share reaches into the tile
            int p = min(s.sharing - 1, (int)((float)start * (float)s.sharing / (float)s.steps));
            while (p > 0 && s.share(p) > start) --p;
            while (s.share(p + 1) <= start) ++p;
            shared = s.share(p) > start || s.share(p + 1) < end;                                            // (else it is all one pair's, which has finished it)
            for (p += member; shared && p < s.sharing && s.share(p) < end; p += 2 * team) {
                // two shares at a time (one that begins with the tile, or before it, has it as its last; one that begins inside it as its first)
                const int p1 = p + team;
                const bool two = p1 < s.sharing && s.share(p1) < end;
                const float *from = a.slots + (((long)(2 * p + (s.share(p) > start ? 0 : 1)) * 2 + block) * a.grad_width + col) * 128 + quad * 32 + lane;
                const float *from1 = a.slots + (((long)(2 * p1 + (s.share(p1) > start ? 0 : 1)) * 2 + block) * a.grad_width + col) * 128 + quad * 32 + lane;
                float t[kJoinCols], t1[kJoinCols];
#pragma unroll
                for (int e = 0; e < kJoinCols; ++e) t[e] = from[e * 128];
                if (two) {
#pragma unroll
                    for (int e = 0; e < kJoinCols; ++e) t1[e] = from1[e * 128];
                }
#pragma unroll
                for (int e = 0; e < kJoinCols; ++e) v[e] += t[e];
                if (two) {
#pragma unroll
                    for (int e = 0; e < kJoinCols; ++e) v[e] += t1[e];
                }
            }
        }
        if (team > 1) {
            float *own = reinterpret_cast<float *>(pieces[warp]);
#pragma unroll
            for (int e = 0; e < kJoinCols; ++e) own[e * 32 + lane] = v[e];
            __syncthreads();
            if (member == 0)
                for (int m = 1; m < team; ++m)
#pragma unroll
                    for (int e = 0; e < kJoinCols; ++e) v[e] += reinterpret_cast<const float *>(pieces[warp + m])[e * 32 + lane];
            __syncthreads();
        }
        if (member == 0 && shared)
            loss_gradient<E>(ptx::smem_u32(pieces[warp]), a, info, loss_row<kLossGrads>(a, (int)info.rows, tile / a.tiles_c * 256 + block * 128 + quad * 32 + lane, dx), dx, tile / a.tiles_c, tile % a.tiles_c, block, quad, col, v);
    }
}

// ---- a few rows
//
// One row is scored as fast as W can be read, by fused multiply-adds in float32 (two a row and pair of elements, beside two conversions: one row over 32000 words of 1024, 66 MB in bfloat16, takes 12 to 16 us, 4 to
// 5.5 TB/s, and the merge behind it 5; two or more are bound by instructions): a tile of a tensor core's product would have 248 empty rows, and float32 inputs would have W read and written once more for their three values.
// A warp takes four words at a time, a lane eight columns of each (kVec: neighbours, 16 bytes a load; else 32 apart); X is in shared memory as float32, where the lanes' pieces of a row lie in
// two sets of 16 bytes so that neighbouring lanes meet no bank conflict.  The 4 R sums are added up over the lanes by exchanges that halve their number (31 for all of 32 sums).
//
// Backward (kG > 0) the same sums give G, so that p = exp(l - lse) has the very logits that lse was formed of: of a row that has learned its label 1 - p is what counts, and another order of addition, the tensor cores',
// put 35 times the error of a plain float32 gradient into it (2 rows over three words of 4032).  Both gradients are then taken from G as of many rows.
constexpr int kFewThreads = 256, kFewWords = 4;
struct LossFew {
    const void *x, *w, *labels;
    int wide, rows, C, V, v0, words;          // words: of V, from v0 on
    long ld_x, ld_w, cap;
    float scale;
    float2 *part;                // [blocks][cap]
    float *chosen;
    // backward
    const float *lse_in, *gm;    // of rows; of packed rows
    uint16_t *g;                 // planes [cap][ld_g]
    long ld_g;
};
__host__ __device__ constexpr size_t few_smem(int R, int C) { return (size_t)R * ((C + 255) / 256 * 256) * sizeof(float); }
template <typename T, int R, bool kVec, int kG>
__global__ void __launch_bounds__(kFewThreads, R <= 2 ? 4 : 2) loss_few_kernel(const LossFew a) {
    extern __shared__ float4 xs[];                            // [R][turns][2][32]
    __shared__ float2 stats[kFewThreads / 32][32];
    ptx::grid_launch();
    ptx::grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, turns = (a.C + 255) / 256;
    // where lane l's i-th column of a turn lies: kVec 256 t + 8 l + i, else 256 t + l + 32 i
    const T *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.w);
    for (int i = threadIdx.x; i < R * turns * 256; i += kFewThreads) {
        const int r = i / (turns * 256), c = i % (turns * 256), t = c >> 8, l = kVec ? c >> 3 & 31 : c & 31, e = kVec ? c & 7 : c >> 5 & 7;
        reinterpret_cast<float *>(xs)[(((r * turns + t) * 2 + (e >> 2)) * 32 + l) * 4 + (e & 3)] = r < a.rows && c < a.C ? to_f32(x[r * a.ld_x + c]) : 0.f;
    }
    constexpr int kSums = kFewWords * R, kSkip = kSums == 32 ? 0 : kSums == 16 ? 1 : kSums == 8 ? 2 : 3;   // lanes that hold the same sum: 2^kSkip
    const int mine = lane >> kSkip, row = mine / kFewWords, word = mine % kFewWords;
    int64_t label = -1;
    if (row < a.rows) label = label_at(a.labels, a.wide, row);
    const float c2 = a.scale * kLossLog2e;
    LossStat stat{-INFINITY, 0.f};
    int labelled = 0, to = -1;                                // backward: rows with a label; this one's place among them, -1: none
    float lse = 0.f, gm = 0.f;
    if constexpr (kG > 0) {
        for (int r = 0; r < a.rows; ++r) {
            const int64_t l = label_at(a.labels, a.wide, r);
            if (l < 0 || l >= a.V) continue;
            if (r == row) to = labelled;
            ++labelled;
        }
        if (to >= 0) { lse = a.lse_in[row]; gm = a.gm[to]; }
        // zeros in the rows up to 64 that the products over rows read, and in the columns up to whole 64 that those over words do
        const int cols = (a.words + 63) / 64 * 8;
        for (int i = blockIdx.x * kFewThreads + threadIdx.x; i < (64 - labelled) * cols; i += gridDim.x * kFewThreads)
#pragma unroll
            for (int h = 0; h < kG; ++h) *reinterpret_cast<uint4 *>(a.g + (h * a.cap + labelled + i / cols) * a.ld_g + i % cols * 8) = make_uint4(0, 0, 0, 0);
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i < labelled * 64; i += kFewThreads)
                if (a.words + i % 64 < 8 * cols)
                    for (int h = 0; h < kG; ++h) a.g[(h * a.cap + i / 64) * a.ld_g + a.words + i % 64] = 0;
    }
    __syncthreads();
    const int groups = (a.words + kFewWords - 1) / kFewWords;
    for (int g = blockIdx.x * (kFewThreads / 32) + warp; g < groups; g += gridDim.x * (kFewThreads / 32)) {
        const T *p[kFewWords];
#pragma unroll
        for (int k = 0; k < kFewWords; ++k) p[k] = w + (long)(a.v0 + min(g * kFewWords + k, a.words - 1)) * a.ld_w;     // (beyond the last word: that again)
        float s[kSums];
#pragma unroll
        for (int i = 0; i < kSums; ++i) s[i] = 0.f;
#pragma unroll 2
        for (int t = 0; t < turns; ++t) {
            const int c = t * 256 + (kVec ? lane * 8 : lane);
            LossEight<T> e[kFewWords];
#pragma unroll
            for (int k = 0; k < kFewWords; ++k) {
                if (kVec) {
                    if (c < a.C) eight_of(p[k] + c, true, 8, e[k]);
                    else
#pragma unroll
                        for (int i = 0; i < (int)sizeof(T) / 2; ++i) e[k].q[i] = make_uint4(0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + 32 * i < a.C) reinterpret_cast<T *>(e[k].q)[i] = p[k][c + 32 * i];
                        else from_f32(reinterpret_cast<T *>(e[k].q)[i], 0.f);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float4 v = xs[((r * turns + t) * 2 + h) * 32 + lane];
#pragma unroll
                    for (int k = 0; k < kFewWords; ++k) {
                        const T *u = reinterpret_cast<const T *>(e[k].q) + 4 * h;
                        float &q = s[r * kFewWords + k];
                        q = fmaf(to_f32(u[0]), v.x, q);
                        q = fmaf(to_f32(u[1]), v.y, q);
                        q = fmaf(to_f32(u[2]), v.z, q);
                        q = fmaf(to_f32(u[3]), v.w, q);
                    }
                }
        }
#pragma unroll
        for (int n = kSums / 2, o = 16; n > 0; n >>= 1, o >>= 1)
#pragma unroll
            for (int i = 0; i < kSums / 2; ++i)
                if (i < n) {
                    const bool up = lane & o;
                    const float other = __shfl_xor_sync(0xffffffffu, up ? s[i] : s[i + n], o);
                    s[i] = (up ? s[i + n] : s[i]) + other;
                }
#pragma unroll
        for (int o = (1 << kSkip) >> 1; o > 0; o >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
        const int v = g * kFewWords + word;
        if constexpr (kG > 0) {
            if (v < a.words && to >= 0 && (lane & ((1 << kSkip) - 1)) == 0) {
                const float d = __fsub_rn(__fmul_rn(s[0], a.scale), lse);
                float q = (a.v0 + v == label ? expm1f(d) : ptx::ex2(d * kLossLog2e)) * gm;
#pragma unroll
                for (int h = 0; h < kG; ++h) {
                    typename std::conditional<std::is_same<T, __half>::value, __half, __nv_bfloat16>::type t;
                    from_f32(t, q);
                    q -= to_f32(t);
                    a.g[(h * a.cap + to) * a.ld_g + v] = *reinterpret_cast<const uint16_t *>(&t);
                }
            }
        } else if (v < a.words) {
            stat = loss_both(stat, LossStat{s[0], 1.f}, c2);
            if (v == label && (lane & ((1 << kSkip) - 1)) == 0) a.chosen[row] = s[0];
        }
    }
    if constexpr (kG > 0) return;
    stats[warp][lane] = make_float2(stat.m, stat.l);
    __syncthreads();
    if ((int)threadIdx.x < a.rows) {
        stat = LossStat{-INFINITY, 0.f};
        for (int u = 0; u < kFewThreads / 32; ++u)
            for (int k = 0; k < kFewWords; ++k) {
                const float2 y = stats[u][(threadIdx.x * kFewWords + k) << kSkip];
                stat = loss_both(stat, LossStat{y.x, y.y}, c2);
            }
        a.part[(long)blockIdx.x * a.cap + threadIdx.x] = make_float2(stat.m, stat.l);
    }
}

// Parts of a row's statistics, joined: 32 rows a block, its warps (as many as the parts keep busy) taking the parts in turn.
constexpr int kMergeWarps = 32;
struct LossMerge {
    const LossInfo *info;
    const float2 *part;
    const float *chosen;
    const int *index;
    long cap;
    int parts;
    float *loss, *lse;
    // rows as they stand (LossArgs): labels, and how many
    const void *labels;
    int wide, V, direct;
    const uint32_t *gave_up;
    uint32_t *status;
    int blocks;
    float scale;
};
__global__ void __launch_bounds__(32 * kMergeWarps) loss_merge_kernel(const LossMerge a) {
    __shared__ float2 shared[kMergeWarps][32];
    ptx::grid_launch();
    ptx::grid_wait();
    const int warps = blockDim.x / 32, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = a.direct ? a.direct : (int)a.info->rows;
    if (a.direct && blockIdx.x == 0 && warp == 0) {
        uint32_t code = 0;
        for (int b = lane; b < a.blocks; b += 32) code = max(code, a.gave_up[b]);
        code = __reduce_max_sync(0xffffffffu, code);
        for (int i = lane; i < (int)(kHeaderBytes / 4); i += 32) a.status[i] = i == 0 ? code : 0;
    }
    const float c2 = a.scale * kLossLog2e;
    for (long r0 = (long)blockIdx.x * 32; r0 < rows; r0 += (long)gridDim.x * 32) {
        const long row = r0 + lane;
        LossStat stat{-INFINITY, 0.f};
        if (row < rows) {
            int p = warp;
            for (; p < a.parts; p += 8 * warps) {
                LossStat s[9];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 x = p + k * warps < a.parts ? a.part[(long)(p + k * warps) * a.cap + row] : make_float2(-INFINITY, 0.f);
                    s[k] = LossStat{x.x, x.y};
                }
                s[8] = stat;
                stat = loss_all(s, c2);
            }
        }
        if (warps > 1) {
            shared[warp][lane] = make_float2(stat.m, stat.l);
            __syncthreads();
        }
        if (warp == 0 && row < rows) {
            for (int w = 1; w < warps; ++w) stat = loss_both(stat, LossStat{shared[w][lane].x, shared[w][lane].y}, c2);
            bool there = true;
            if (a.direct) {
                const int64_t label = label_at(a.labels, a.wide, row);
                there = label >= 0 && label < a.V;
            }
            const long n = a.direct ? row : a.index[row];
            a.loss[n] = there ? loss_of(stat, a.chosen[row], a.scale) : 0.f;
            a.lse[n] = there ? loss_lse(stat, a.scale) : 0.f;
        }
        if (warps > 1) __syncthreads();
    }
}

}  // namespace flare
