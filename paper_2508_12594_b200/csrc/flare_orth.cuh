// Orthogonalising an update by Newton-Schulz products:  X0 = U / (|U|_F + eps),  then `steps` times
//
//     A = X X^T,   B = a I + b A + c A^2,   X <- B X                      (the odd quintic a x + b x^3 + c x^5 of the singular values)
//
// with X [S, L], S the short side (U transposed where it is tall).  The quintic lifts small singular values by up to a^steps (485 for
// the usual coefficients), and with them whatever was rounded away of X beside its large ones: bfloat16 or tf32 factors (8, 11 bits)
// are off by several percent after five steps on matrices with a few strong directions.  So every factor is carried as two float16
// halves (22 bits), x = hi + lo at a power-of-two scale that keeps lo a normal number, and a product is hi hi + hi lo + lo hi on the
// tensor cores with float32 sums: three products at the 16-bit rate against one at a rate some twenty times lower in float32.
// A, B and the squares are symmetric: pairs of blocks compute only the tiles on and above the diagonal and store each twice, teams where that is the
// faster form (team_plan); clusters and single blocks compute both halves.
#pragma once

#include "flare_common.cuh"
#include "flare_ptx.cuh"

namespace flare {

// What a step's products are for.
enum { kOrthGram = 0, kOrthPoly = 1, kOrthApply = 2, kOrthLast = 3 };
// 64-deep steps whose sums stay in tensor memory, which adds with truncation, before they are added up in registers, rounded (see the large matrices).
__host__ __device__ constexpr int orth_chunk(int kind) { return kind == kOrthGram ? 8 : 4; }

// The matrices that go in and come out, and the update of the weights around them (m != nullptr).
struct OrthOuter {
    const void *g;               // [count] matrices [rows, cols], rows ld_g and matrices step_g apart
    void *out;                   // the orthogonalised ones, or the new weights
    const void *w;
    const float *m;
    float *m_out;
    long ld_g, step_g, ld_out, step_out;
    int rows, cols, g_type, out_type;
    int tall;                    // rows > cols: X is the transpose
    int in_fours, out_fours;     // four columns at a time: widths, strides and pointers allow it
    int nesterov;
    float momentum, keep, rate;  // w' = keep w - rate O
    float eps;
};

// f(element of the type that is chosen at run time, FLARE_DTYPE_*)
template <typename F>
__device__ __forceinline__ void with_type(int type, F f) {
    if (type == 0) f(float{});
    else if (type == 1) f(__nv_bfloat16{});
    else f(__half{});
}
// V (1 or 4) neighbouring elements.
template <int V, typename E>
__device__ __forceinline__ void load_v(const E *p, float (&v)[V]) {
    if constexpr (V == 1) v[0] = to_f32(*p);
    else if constexpr (sizeof(E) == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(p);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
        const uint2 q = *reinterpret_cast<const uint2 *>(p);
        E e[4];
        *reinterpret_cast<uint2 *>(e) = q;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_f32(e[i]);
    }
}
template <int V, typename E>
__device__ __forceinline__ void store_v(E *p, const float (&v)[V]) {
    if constexpr (V == 1) from_f32(*p, v[0]);
    else if constexpr (sizeof(E) == 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else {
        __align__(8) E e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) from_f32(e[i], v[i]);
        *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(e);
    }
}

// A thread's walk over the groups of V columns of a matrix, `step` at a time, without divisions.
struct OrthWalk {
    int r, c, dr, dc, groups;
    __device__ __forceinline__ OrthWalk(uint32_t first, uint32_t step, int groups_) : groups(groups_) {
        r = (int)(first / (uint32_t)groups); c = (int)(first % (uint32_t)groups);
        dr = (int)(step / (uint32_t)groups); dc = (int)(step % (uint32_t)groups);
    }
    __device__ __forceinline__ void next() {
        r += dr; c += dc;
        if (c >= groups) { c -= groups; ++r; }
    }
};
// use(r, c, V values) for every group of columns of the walk from `first`, of what is orthogonalised.  kNew: the momentum has been updated already.
// kBatch groups are asked for before the first is used: one at a time, with a store between two loads that the compiler must keep in order, each
// costs a round trip to memory.
template <int V, typename G, bool kMomentum, bool kNew, int kBatch, typename F>
__device__ __forceinline__ void orth_elements_as(const OrthOuter &o, size_t mat, uint32_t first, uint32_t step, F use) {
    OrthWalk walk(first, step, o.cols / V);
    const G *g = static_cast<const G *>(o.g) + mat * o.step_g;
    const size_t base = mat * (size_t)o.rows * o.cols;
    while (walk.r < o.rows) {
        int r[kBatch], c[kBatch];
        float u[kBatch][V], m[kBatch][V];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            r[k] = walk.r; c[k] = walk.c * V;
            if (walk.r < o.rows) {
                load_v<V>(g + (size_t)r[k] * o.ld_g + c[k], u[k]);
                if constexpr (kMomentum) load_v<V>((kNew ? o.m_out : o.m) + base + (size_t)r[k] * o.cols + c[k], m[k]);
            }
            walk.next();
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (r[k] >= o.rows) break;
            if constexpr (kMomentum) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (!kNew) m[k][i] = fmaf(o.momentum, m[k][i], (1.f - o.momentum) * u[k][i]);
                    u[k][i] = o.nesterov ? fmaf(o.momentum, m[k][i], (1.f - o.momentum) * u[k][i]) : m[k][i];
                }
                if (!kNew) store_v<V>(o.m_out + base + (size_t)r[k] * o.cols + c[k], m[k]);
            }
            use(r[k], c[k], u[k]);
        }
    }
}
template <bool kNew, typename F>
__device__ __forceinline__ void orth_elements(const OrthOuter &o, size_t mat, uint32_t first, uint32_t step, F use) {
    with_type(o.g_type, [&](auto type) {
        using G = decltype(type);
        if (o.in_fours) {
            if (o.m) orth_elements_as<4, G, true, kNew, 4>(o, mat, first, step, use);
            else orth_elements_as<4, G, false, kNew, 4>(o, mat, first, step, use);
        } else {
            if (o.m) orth_elements_as<1, G, true, kNew, 8>(o, mat, first, step, use);
            else orth_elements_as<1, G, false, kNew, 8>(o, mat, first, step, use);
        }
    });
}
// Writes the result, V columns of a row at a time: get(r, c, V values of O).
template <int V, typename E, int kBatch, typename F>
__device__ __forceinline__ void orth_results_as(const OrthOuter &o, size_t mat, uint32_t first, uint32_t step, F get) {
    OrthWalk walk(first, step, o.cols / V);
    E *out = static_cast<E *>(o.out) + mat * o.step_out;
    const E *w = o.w ? static_cast<const E *>(o.w) + mat * o.step_out : nullptr;
    while (walk.r < o.rows) {
        int r[kBatch], c[kBatch];
        float old[kBatch][V];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            r[k] = walk.r; c[k] = walk.c * V;
            if (w && walk.r < o.rows) load_v<V>(w + (size_t)r[k] * o.ld_out + c[k], old[k]);
            walk.next();
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (r[k] >= o.rows) break;
            float v[V];
            get(r[k], c[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (w) v[i] = fmaf(-o.rate, v[i], o.keep * old[k][i]);
            store_v<V>(out + (size_t)r[k] * o.ld_out + c[k], v);
        }
    }
}
template <typename F>
__device__ __forceinline__ void orth_results(const OrthOuter &o, size_t mat, uint32_t first, uint32_t step, F get) {
    with_type(o.out_type, [&](auto type) {
        using E = decltype(type);
        if (o.out_fours) orth_results_as<4, E, 4>(o, mat, first, step, get);
        else orth_results_as<1, E, 8>(o, mat, first, step, get);
    });
}

__device__ __forceinline__ void split_half(float v, __half &hi, __half &lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}
// Eight values to their packed halves.
__device__ __forceinline__ void split8(const float *v, uint4 &hi, uint4 &lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 a = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        const float2 f = __half22float2(a);
        const __half2 b = __floats2half2_rn(v[2 * i] - f.x, v[2 * i + 1] - f.y);
        h[i] = *reinterpret_cast<const uint32_t *>(&a);
        l[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void join8(uint4 hi, uint4 lo, float *v) {
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&h[i])), b = __half22float2(*reinterpret_cast<const __half2 *>(&l[i]));
        v[2 * i] = a.x + b.x;
        v[2 * i + 1] = a.y + b.y;
    }
}

// Power-of-two scales of the halves (from the quintic's range, see orth_scales) and the coefficients.
struct OrthScales { float x, a, b; float ca, cb, cc; };

// Clears the workspace header and the counters behind it.
__global__ void __launch_bounds__(256) orth_clear_kernel(uint32_t *words, int n) {
    ptx::grid_launch();
    ptx::grid_wait();
    for (int i = threadIdx.x; i < n; i += 256) words[i] = 0u;
}

// ---------------------------------------------------------------- norm and first split, for matrices that do not fit a block
constexpr int kOrthNormThreads = 256;

// Momentum, and per block the sum of squares of its share of a matrix, in float64 (with eps = 0 gradients of 1e-25 are as good as any).  Grid (blocks, count).
__global__ void __launch_bounds__(kOrthNormThreads) orth_norm_kernel(OrthOuter o, double *part) {
    ptx::grid_launch();
    ptx::grid_wait();
    double sum = 0.0;
    orth_elements<false>(o, blockIdx.y, blockIdx.x * kOrthNormThreads + threadIdx.x, gridDim.x * kOrthNormThreads, [&](int, int, const auto &u) {
        for (float x : u) sum += (double)x * x;
    });
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
    __shared__ double sh[kOrthNormThreads / 32];
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kOrthNormThreads / 32; ++k) sum += sh[k];
        part[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
    }
}

__device__ __forceinline__ uint32_t half_pair(float a, float b, uint32_t &lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(a - f.x, b - f.y);
    lo = *reinterpret_cast<const uint32_t *>(&l);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// The halves of X0, [2 count][S][ld] (high and low of a matrix in turn), from the `parts` partial sums of squares: this block's share (the `member`-th
// of `members`).  tall: tiles of 64 x 64 through shared memory, 64 x 65 floats at `tile`.  sh: room for a double.  All threads of the block.
__device__ __forceinline__ void orth_split(const OrthOuter &o, size_t mat, const double *part, int parts, __half *x, long ld, float scale, float *tile, double *sh,
                                           int member, int members) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    __syncthreads();
    if (warp == 0) {
        double sum = 0.0;
        for (int i = lane; i < parts; i += 32) sum += __ldcg(part + i);
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        if (lane == 0) *sh = (double)scale / (sqrt(sum) + (double)o.eps);
    }
    __syncthreads();
    const double f = *sh;
    const int S = o.tall ? o.cols : o.rows, L = o.tall ? o.rows : o.cols;
    __half *hi = x + 2 * mat * S * ld, *lo = hi + S * ld;
    if (!o.tall) {
        orth_elements<true>(o, mat, member * blockDim.x + threadIdx.x, members * blockDim.x, [&](int r, int c, const auto &u) {
            constexpr int V = sizeof(u) / sizeof(float);
            const size_t at = (size_t)r * ld + c;
            if constexpr (V == 1) split_half((float)(u[0] * f), hi[at], lo[at]);
            else {
                uint2 h, l;
                h.x = half_pair((float)(u[0] * f), (float)(u[1] * f), l.x);
                h.y = half_pair((float)(u[2] * f), (float)(u[3] * f), l.y);
                *reinterpret_cast<uint2 *>(hi + at) = h;
                *reinterpret_cast<uint2 *>(lo + at) = l;
            }
        });
        return;
    }
    const int tiles_c = (o.cols + 63) / 64, tiles = tiles_c * ((o.rows + 63) / 64);
    for (int t = member; t < tiles; t += members) {
        const int r0 = t / tiles_c * 64, c0 = t % tiles_c * 64;
        with_type(o.g_type, [&](auto type) {
            using G = decltype(type);
            const G *g = static_cast<const G *>(o.g) + mat * o.step_g;
            const float *m = o.m ? o.m_out + mat * (size_t)o.rows * o.cols : nullptr;
            for (int i0 = threadIdx.x; i0 < 4096; i0 += 8 * blockDim.x) {
                float u[8], q[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = i0 + k * blockDim.x, r = r0 + (i >> 6), c = c0 + (i & 63);
                    const bool yes = i < 4096 && r < o.rows && c < o.cols;
                    u[k] = yes ? to_f32(g[(size_t)r * o.ld_g + c]) : 0.f;
                    q[k] = yes && m ? m[(size_t)r * o.cols + c] : 0.f;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = i0 + k * blockDim.x;
                    if (i < 4096) tile[(i >> 6) * 65 + (i & 63)] = !m ? u[k] : o.nesterov ? fmaf(o.momentum, q[k], (1.f - o.momentum) * u[k]) : q[k];
                }
            }
        });
        __syncthreads();
        const int l = r0 + 2 * lane;
        for (int s = warp; s < 64; s += warps)
            if (c0 + s < S && l < L) {                               // (ld is even; what is beyond the last column is never read)
                uint32_t low;
                const uint32_t high = half_pair((float)(tile[2 * lane * 65 + s] * f), (float)(tile[(2 * lane + 1) * 65 + s] * f), low);
                const size_t at = (size_t)(c0 + s) * ld + l;
                *reinterpret_cast<uint32_t *>(hi + at) = high;
                *reinterpret_cast<uint32_t *>(lo + at) = low;
            }
        __syncthreads();
    }
}
__global__ void __launch_bounds__(256) orth_split_kernel(OrthOuter o, const double *part, int parts, __half *x, long ld, float scale) {
    __shared__ float tile[64 * 65];
    __shared__ double sh;
    ptx::grid_launch();
    ptx::grid_wait();
    orth_split(o, blockIdx.y, part + (size_t)blockIdx.y * parts, parts, x, ld, scale, tile, &sh, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------- one product
// Instruction descriptor for kind::f16 with float16 operands and float accumulation.
__host__ __device__ constexpr uint32_t instr_desc_f16(int m, int n, int b_mn) {
    return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

struct OrthProduct {
    const __half *a;             // halves of A (kOrthPoly) [2 count][S][ld_a]
    long ld_a;
    int S, N, K;                 // result [S, N], sums over K
    int tiles_m, tiles_n, tiles; // tiles of a matrix, down, across and in all
    float per_m;                 // 1 / tiles_m
    int width;                   // columns of a tile: 256 of a pair's, 128 or 64 of a single block's
    int upper;                   // a symmetric result: tiles on and above the diagonal, each stored twice
    float f, fa, fi;             // result = f sums (+ fa A + fi I)
};
// A matrix of halves in the three forms its tiles are moved in: loaded (64 x 64), stored (32 rows of 64), stored transposed (64 rows of 32).
struct HalfMaps { CUtensorMap load, store, store_t; };

// Warp 0 loads, warp 1 issues, warps 4 to 11 take the sums out of tensor memory.
constexpr int kOrthThreads = 384, kOrthStages = 3;
constexpr uint32_t kOrthHalfTile = 128 * 128;                       // bytes: 128 rows (or 64 rows of two blocks of columns) of 64 float16
constexpr uint32_t kOrthStage = 4 * kOrthHalfTile;                  // A high, A low, B high, B low
constexpr uint32_t kOrthPiece = 4096;                               // a warp's piece of the result on its way out: 32 x 64 halves, 32 x 32 floats
constexpr size_t kOrthSmem = 1024 + kOrthStages * kOrthStage + 8 * kOrthPiece + 256;

// The tile (i, j), i <= j, that comes t-th row by row.
__device__ __forceinline__ void upper_tile(int t, int n, int &i, int &j) {
    i = 0;
    while (t >= n - i) { t -= n - i; ++i; }
    j = i + t;
}

namespace ptx {
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// kPair = 2: the two blocks of a cluster as one (256 rows, each block's 128 in its own tensor memory; each block holds half of B).
template <int kPair> __device__ __forceinline__ void tmem_alloc_for(uint32_t slot, uint32_t cols) {
    if (kPair == 1) { tmem_alloc(slot, cols); return; }
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
template <int kPair> __device__ __forceinline__ void tmem_dealloc_for(uint32_t taddr, uint32_t cols) {
    if (kPair == 1) tmem_dealloc(taddr, cols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
template <int kPair> __device__ __forceinline__ void tma_load_3d_for(uint32_t dst, const CUtensorMap *m, uint32_t bar, int c0, int c1, int c2) {
    if (kPair == 1) { tma_load_3d(dst, m, bar, c0, c1, c2); return; }
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
template <int kPair> __device__ __forceinline__ void mma_ss_for(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (kPair == 1) { mma_ss(d, a, b, idesc, accumulate); return; }
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"(accumulate)
                 : "memory");
}
// (kPair = 2: the barriers of both blocks)
template <int kPair> __device__ __forceinline__ void mma_commit_for(uint32_t bar) {
    if (kPair == 1) { mma_commit(bar); return; }
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
}  // namespace ptx

// A warp's 32 rows x 32 columns of the result, one row a lane, into the output (rows s0.., columns l0..) by way of shared memory, so that
// neighbouring lanes write neighbouring elements whichever way the output lies.  buf: 4096 bytes of the warp's own.
template <typename E>
__device__ __forceinline__ void outer_piece(const OrthOuter &o, size_t mat, int s0, int l0, int S, int L, const float *v, float f, float *buf) {
    const int lane = threadIdx.x & 31;
    // k: the other dimension of the piece; a lane's element of it is at + k ld_out
    const int r0 = o.tall ? l0 : s0, c = (o.tall ? s0 : l0) + lane, rows = c < (o.tall ? S : L) ? min(32, (o.tall ? L : S) - r0) : 0;
    E *out = static_cast<E *>(o.out) + mat * o.step_out + (size_t)r0 * o.ld_out + c;
    const E *w = o.w ? static_cast<const E *>(o.w) + mat * o.step_out + (size_t)r0 * o.ld_out + c : nullptr;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 32; ++k) buf[lane * 32 + (k ^ lane)] = v[k];
    __syncwarp();
    // (from here on without v's registers, in loops that are not unrolled over the whole piece: the other pieces' sums are still in theirs)
#pragma unroll 1
    for (int k0 = 0; k0 < rows; k0 += 16) {
        float x[16];
        if (w) {
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] = k0 + k < rows ? to_f32(w[k * o.ld_out]) : 0.f;
            w += 16 * o.ld_out;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float y = f * buf[o.tall ? lane * 32 + ((k0 + k) ^ lane) : (k0 + k) * 32 + (lane ^ (k0 + k))];
            x[k] = w ? fmaf(-o.rate, y, o.keep * x[k]) : y;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (k0 + k < rows) from_f32(out[k * o.ld_out], x[k]);
        out += 16 * o.ld_out;
    }
    __syncwarp();
}

// Barriers and tensor memory of a block's pipeline, and how far it has come: stages loaded or issued, sets of sums handed over (each role
// counts for itself).
struct OrthPipe {
    uint32_t smem0, pieces0, bars, tmem;
    uint8_t *smem;
    volatile uint32_t *abort_flag;
    uint32_t n, c;
    __device__ __forceinline__ uint32_t full(uint32_t s) const { return bars + 8 * s; }
    __device__ __forceinline__ uint32_t empty(uint32_t s) const { return bars + 8 * (kOrthStages + s); }
    __device__ __forceinline__ uint32_t acc_full(uint32_t b) const { return bars + 8 * (2 * kOrthStages + b); }
    __device__ __forceinline__ uint32_t acc_empty(uint32_t b) const { return bars + 8 * (2 * kOrthStages + 2 + b); }
};
// What this block (or pair) does of a product: tiles t0, t0 + step .. of `total` (all matrices from `mat` on), the steps kb0 .. kb1 along K of each.
struct OrthShare { int t0, step, total, mat, kb0, kb1; };
struct OrthTile { int mat, i, j; };
__device__ __forceinline__ bool orth_symmetric(int kind) { return kind == kOrthGram || kind == kOrthPoly; }
__device__ __forceinline__ OrthTile orth_tile(const OrthProduct &p, const OrthShare &w, int t) {
    OrthTile x;
    x.mat = w.mat;
    if (t >= p.tiles) {
        const int more = t / p.tiles;
        x.mat += more;
        t -= more * p.tiles;
    }
    if (p.upper) upper_tile(t, p.tiles_n, x.i, x.j);
    else {                                                   // (a division, for numbers of tiles: t + 1/2 over tiles_m is never near a whole number)
        x.j = (int)(((float)t + 0.5f) * p.per_m);
        x.i = t - x.j * p.tiles_m;
    }
    return x;
}

// Sets the pipeline up; all threads of the block.
template <int kPair>
__device__ __forceinline__ OrthPipe orth_pipe(uint8_t *raw, uint32_t *tmem_slot, volatile uint32_t *abort_flag) {
    OrthPipe q;
    q.smem = ptx::align_1024(raw);
    q.smem0 = ptx::smem_u32(q.smem);
    q.pieces0 = q.smem0 + kOrthStages * kOrthStage;
    q.bars = q.pieces0 + 8 * kOrthPiece;
    q.abort_flag = abort_flag;
    q.n = q.c = 0;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < kOrthStages; ++s) { ptx::mbar_init(q.full(s), 1); ptx::mbar_init(q.empty(s), 1); }
        for (int b = 0; b < 2; ++b) { ptx::mbar_init(q.acc_full(b), 1); ptx::mbar_init(q.acc_empty(b), 8 * kPair); }
        ptx::fence_mbar_init();
    }
    if (ptx::warp_index() == 1) ptx::tmem_alloc_for<kPair>(ptx::smem_u32(tmem_slot), 256 * kPair);
    ptx::tc_fence_before();
    __syncthreads();
    if (kPair == 2) ptx::cluster_meet();
    ptx::tc_fence_after();
    q.tmem = *tmem_slot;
    return q;
}
// What a block that gave up a wait has asked for, copies into its shared memory and products into its tensor memory, may still be on its way, and
// which of its barriers would say so is not known then: it is given a millisecond, some hundred times what it takes, before the block ends.
__device__ __forceinline__ void let_arrive(volatile uint32_t *abort_flag) {
    if (*abort_flag == 0) return;
    for (const uint64_t t0 = ptx::globaltimer_ns(); ptx::globaltimer_ns() - t0 < 1000000ull;) __nanosleep(2000);
}
template <int kPair>
__device__ __forceinline__ void orth_pipe_end(const OrthPipe &q, uint32_t *status) {
    ptx::tc_fence_before();
    __syncthreads();
    let_arrive(q.abort_flag);
    if (kPair == 2) ptx::cluster_meet();                                 // (nobody's shared or tensor memory is needed any more)
    if (threadIdx.x == 0 && *q.abort_flag != 0) *status = *q.abort_flag;
    if (ptx::warp_index() == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_for<kPair>(q.tmem, 256 * kPair);
    }
}

// The loading warp's part.  ta: rows of the left factor; tb: rows of the right one's transpose (kOrthGram, kOrthPoly: sums along rows) or the right
// one's own rows.
template <int kPair>
__device__ __forceinline__ void orth_load(OrthPipe &q, const OrthProduct &p, const OrthShare &w, int kind, const CUtensorMap *ta, const CUtensorMap *tb) {
    const bool symmetric = orth_symmetric(kind);
    if (!ptx::elect_one()) return;
    const int in_pair = kPair == 2 ? (int)(blockIdx.x & 1) : 0;
    asm volatile("fence.proxy.async.global;" ::: "memory");              // (what was stored by others before this, for the loads by TMA)
    for (int t = w.t0; t < w.total; t += w.step) {
        const OrthTile x = orth_tile(p, w, t);
        const bool own = symmetric && x.i == x.j && (kPair == 2 || p.width == 128);   // both factors are the same rows
        const int ra = x.i * 128 * kPair + in_pair * 128, rb = kPair == 2 ? x.j * 256 + in_pair * 128 : x.j * p.width, right = kPair == 2 ? 128 : p.width;
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++q.n) {
            const uint32_t s = q.n % kOrthStages;
            if (q.n >= kOrthStages && !ptx::mbar_wait(q.empty(s), (q.n / kOrthStages - 1) & 1, q.abort_flag, 101)) return;
            const uint32_t at = q.smem0 + s * kOrthStage, bar = kPair == 2 ? ptx::in_block(q.full(s), 0) : q.full(s);
            if (in_pair == 0) ptx::mbar_arrive_expect_tx(q.full(s), kPair * 2 * (kOrthHalfTile + (own ? 0 : right * 128)));
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    ptx::tma_load_3d_for<kPair>(at + h * kOrthHalfTile + r * 8192, ta, bar, kb * 64, ra + r * 64, 2 * x.mat + h);
                    if (own || r * 64 >= right) continue;
                    if (symmetric) ptx::tma_load_3d_for<kPair>(at + (2 + h) * kOrthHalfTile + r * 8192, tb, bar, kb * 64, rb + r * 64, 2 * x.mat + h);
                    else ptx::tma_load_3d_for<kPair>(at + (2 + h) * kOrthHalfTile + r * 8192, tb, bar, rb + r * 64, kb * 64, 2 * x.mat + h);
                }
        }
    }
}

// The issuing warp's part (of a pair: its first block's).
template <int kPair>
__device__ __forceinline__ void orth_issue(OrthPipe &q, const OrthProduct &p, const OrthShare &w, int kind) {
    const bool symmetric = orth_symmetric(kind);
    constexpr int kTileN = 128 * kPair;
    constexpr uint32_t hi = ptx::desc_hi(1024, 2), low = kOrthHalfTile >> 4;
    const uint32_t idesc = instr_desc_f16(128 * kPair, kPair == 2 ? 256 : p.width, symmetric ? 0 : 1), b_lbo = symmetric ? 16 : 8192, b_step = (symmetric ? 32 : 2048) >> 4;
    if (!ptx::elect_one()) return;
    for (int t = w.t0; t < w.total; t += w.step) {
        const OrthTile x = orth_tile(p, w, t);
        const bool own = symmetric && x.i == x.j && (kPair == 2 || p.width == 128);
        for (int kb = w.kb0; kb < w.kb1; ++q.c) {
            const uint32_t acc = q.tmem + (q.c & 1) * kTileN;
            if (q.c >= 2 && !ptx::mbar_wait(q.acc_empty(q.c & 1), (q.c / 2 - 1) & 1, q.abort_flag, 102)) return;
            ptx::tc_fence_after();
            for (int k1 = min(kb + orth_chunk(kind), w.kb1), first = 1; kb < k1; ++kb, ++q.n, first = 0) {
                const uint32_t s = q.n % kOrthStages;
                if (!ptx::mbar_wait(q.full(s), (q.n / kOrthStages) & 1, q.abort_flag, 103)) return;
                ptx::tc_fence_after();
                const uint32_t at = q.smem0 + s * kOrthStage;
                const uint32_t a0 = ptx::desc_lo(at, 16), b0 = ptx::desc_lo(own ? at : at + 2 * kOrthHalfTile, b_lbo);
                const int deep = min(4, (p.K - kb * 64 + 15) / 16);           // (what lies beyond K is zeros)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k >= deep) break;
                    const uint32_t a = a0 + k * 2, b = b0 + k * b_step;
                    ptx::mma_ss_for<kPair>(acc, ptx::desc(a + low, hi), ptx::desc(b, hi), idesc, !first || k > 0);
                    ptx::mma_ss_for<kPair>(acc, ptx::desc(a, hi), ptx::desc(b + low, hi), idesc, 1);
                    ptx::mma_ss_for<kPair>(acc, ptx::desc(a, hi), ptx::desc(b, hi), idesc, 1);
                }
                ptx::mma_commit_for<kPair>(q.empty(s));
            }
            ptx::mma_commit_for<kPair>(q.acc_full(q.c & 1));
        }
    }
}

// The result warps' parts.  First a tile's sums into registers, a row a thread and half of the tile's columns (mine: this warp has columns): false if a
// wait gave up.
template <int kPair>
__device__ __forceinline__ bool orth_sums(OrthPipe &q, int chunks, float (&v)[64 * kPair], bool mine = true) {
    constexpr int kTileN = 128 * kPair, kCols = 64 * kPair;
    const int warp = ptx::warp_index(), quad = warp & 3, half = (warp - 4) >> 2, lane = threadIdx.x & 31;
    const uint32_t acc = q.tmem + ((uint32_t)(quad * 32) << 16) + half * kCols;
    for (int i = 0; i < chunks; ++i, ++q.c) {
        const bool ok = ptx::mbar_wait(q.acc_full(q.c & 1), (q.c / 2) & 1, q.abort_flag, 104);
        if (!__all_sync(0xffffffffu, ok)) return false;
        ptx::tc_fence_after();
#pragma unroll
        for (int k = 0; k < kCols; k += 32) {
            if (!mine) break;
            uint32_t u[32];
            ptx::tmem_ld32(acc + (q.c & 1) * kTileN + k, u);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) v[k + e] = i == 0 ? __uint_as_float(u[e]) : v[k + e] + __uint_as_float(u[e]);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (kPair == 2) ptx::mbar_arrive_cluster(ptx::in_block(q.acc_empty(q.c & 1), 0));
            else ptx::mbar_arrive(q.acc_empty(q.c & 1));
        }
    }
    return true;
}
// Then what they are for: kCols columns from col0 on of the warp's 32 rows from row0 on; mirror: the tile's transpose is stored too.
// The part of A that the result's 32 rows x 64 columns want, eight lanes a row: neighbouring lanes next to each other (a row a lane, as the sums lie, would
// ask for 32 lines at a time).
struct OrthPart { uint4 h[8], l[8]; };
__device__ __forceinline__ void orth_part(const OrthProduct &p, int mat, int row0, int col0, OrthPart &a) {
    const int lane = threadIdx.x & 31, col = col0 + (lane & 7) * 8;
    const long plane = (long)p.S * p.ld_a;
    const __half *at = p.a + 2 * mat * plane + (long)(row0 + (lane >> 3)) * p.ld_a + col;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        a.h[e] = a.l[e] = make_uint4(0, 0, 0, 0);
        if (row0 + 4 * e + (lane >> 3) < p.S && col < p.N) {
            a.h[e] = __ldcg(reinterpret_cast<const uint4 *>(at + (long)4 * e * p.ld_a));   // (stored by other blocks of this very launch, it may be)
            a.l[e] = __ldcg(reinterpret_cast<const uint4 *>(at + plane + (long)4 * e * p.ld_a));
        }
    }
}
// Through shared memory to a row a lane: v <- f v + fa A, one half at a time.
__device__ __forceinline__ void orth_part_add(uint32_t piece, const OrthProduct &p, const OrthPart &a, float *v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint4 &x = half ? a.l[e] : a.h[e];
            const uint32_t r[4] = {x.x, x.y, x.z, x.w};
            const int row = 4 * e + (lane >> 3);
            ptx::sts128(piece + row * 128 + (((lane & 7) ^ (row & 7)) << 4), r);
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float4 x = ptx::lds128(piece + lane * 128 + ((e ^ (lane & 7)) << 4));
            const uint32_t r[4] = {__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(x.z), __float_as_uint(x.w)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&r[i]));
                float &v0 = v[8 * e + 2 * i], &v1 = v[8 * e + 2 * i + 1];
                v0 = fmaf(p.fa, y.x, half ? v0 : p.f * v0);
                v1 = fmaf(p.fa, y.y, half ? v1 : p.f * v1);
            }
        }
    }
    __syncwarp();
}
// kRoomy: the stages are free (this is the block's only tile of the product), so that each piece has a place of its own and none waits for another.
template <bool kRoomy, typename E, int kCols>
__device__ __forceinline__ void orth_finish(const OrthPipe &q, const OrthProduct &p, const OrthOuter &o, int kind, int mat, int row0, int col0, bool mirror,
                                            const CUtensorMap *out, const CUtensorMap *out_t, float (&v)[kCols]) {
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31, row = row0 + lane;
    const uint32_t piece = kRoomy ? q.smem0 + (warp - 4) * 4 * kOrthPiece : q.pieces0 + (warp - 4) * kOrthPiece;
    uint8_t *piece_p = q.smem + kOrthStages * kOrthStage + (warp - 4) * kOrthPiece;
    if (kind == kOrthLast) {
#pragma unroll
        for (int k = 0; k < kCols; k += 32)
            if (row0 < p.S && col0 + k < p.N) outer_piece<E>(o, mat, row0, col0 + k, p.S, p.N, v + k, p.f, reinterpret_cast<float *>(piece_p));
        return;
    }
#pragma unroll
    for (int k = 0; k < kCols; k += 64) {
        if (row0 >= p.S || col0 + k >= p.N) continue;                    // (uniform over the warp)
        if (kind == kOrthPoly) {
            OrthPart part;
            orth_part(p, mat, row0, col0 + k, part);
            if (!kRoomy) {                                               // (the piece is on its way out)
                if (lane == 0) ptx::tma_store_wait<true>();
            }
            orth_part_add(q.pieces0 + (warp - 4) * kOrthPiece, p, part, v + k);
            if (row0 < col0 + k + 64 && col0 + k < row0 + 32) {
#pragma unroll
                for (int e = 0; e < 64; ++e) v[k + e] += row == col0 + k + e ? p.fi : 0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 64; ++e) v[k + e] *= p.f;
        }
        uint4 half[2][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) split8(v + k + 8 * e, half[0][e], half[1][e]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // 32 rows of 64 columns, 128-byte swizzle
            uint32_t at = piece + (kRoomy ? (2 * h) * kOrthPiece : 0);
            if (!kRoomy) {
                if (lane == 0) ptx::tma_store_wait<true>();
                __syncwarp();
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t r[4] = {half[h][e].x, half[h][e].y, half[h][e].z, half[h][e].w};
                ptx::sts128(at + lane * 128 + ((e ^ (lane & 7)) << 4), r);
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                ptx::tma_store_3d(out, at, col0 + k, row0, 2 * mat + h);
                ptx::tma_store_commit();
            }
            if (!mirror) continue;
            // the same 64 columns as rows of 32: 64-byte swizzle
            if (!kRoomy) {
                if (lane == 0) ptx::tma_store_wait<true>();
                __syncwarp();
            } else {
                at += kOrthPiece;
            }
#pragma unroll
            for (int e = 0; e < 64; ++e) {
                const uint32_t word = (&half[h][e / 8].x)[(e / 2) & 3], x = e & 1 ? word >> 16 : word;
                asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + e * 64 + (((lane >> 3) ^ ((e >> 1) & 3)) << 4) + (lane & 7) * 2), "h"((uint16_t)x) : "memory");
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                ptx::tma_store_3d(out_t, at, row0, col0 + k, 2 * mat + h);
                ptx::tma_store_commit();
            }
        }
    }
}
template <int kPair, typename E>
__device__ __forceinline__ void orth_results_of(OrthPipe &q, const OrthProduct &p, const OrthShare &w, const OrthOuter &o, int kind, const CUtensorMap *out,
                                                const CUtensorMap *out_t) {
    constexpr int kTileN = 128 * kPair, kCols = 64 * kPair;
    const int warp = ptx::warp_index(), quad = warp & 3, half = (warp - 4) >> 2, in_pair = kPair == 2 ? (int)(blockIdx.x & 1) : 0;
    const int chunks = (w.kb1 - w.kb0 + orth_chunk(kind) - 1) / orth_chunk(kind);
    for (int t = w.t0; t < w.total; t += w.step) {
        const OrthTile x = orth_tile(p, w, t);
        float v[kCols];
        if (!orth_sums<kPair>(q, chunks, v)) break;
        orth_finish<false, E>(q, p, o, kind, x.mat, x.i * kTileN + in_pair * 128 + quad * 32, x.j * kTileN + half * kCols, p.upper && x.i != x.j, out, out_t, v);
    }
    if ((threadIdx.x & 31) == 0) ptx::tma_store_wait<false>();
    __syncwarp();
}

// ---- large matrices: a launch per product, tiles of 256 x 256 by pairs of blocks
//
// Tensor memory adds with truncation, which over K = 4096 (768 additions of 16 products) is off by 2e-5 of a sum of equal signs.  So sums stay there for
// some steps only (orth_chunk) and are added up in registers, rounded, while the next ones run in a second set of columns.  Of the squares and of B X it
// is four (K = 256): with eight, as X X^T has them, whose error hardly matters, the result's 2-norm is off by 2.4e-5 instead of 1.2e-5 (1003 x 2601)
// and 1.5e-5 instead of 7.4e-6 (four of 2048 x 2048), single entries by up to 2.3e-4 of the RMS instead of 1.4e-4.  It costs 2 % (2048 x 2048 462 us
// instead of 452, two of 4096 x 4096 6900 instead of 6790) and up to 5 (four of 1024 x 1024 293 instead of 279); two steps: half the error again, 10 % more.
// (The same second set lets a tile's results go out under the next tile's products.)
// 256 x 256 x 64 of two halves each is 64 KB a block and stage, three stages; a pair reads half of what two blocks of 128 x 256 would.  Bound by the tensor
// pipe: an update of 2 x 4096 x 4096 (2.75 TFLOP, three products of each) takes 7.0 to 7.3 ms, 1130 to 1180 TFLOP/s, the pipe 87 (squares) to 97 % (B X)
// busy, the clock under the power limit.
struct OrthPairArgs {
    OrthProduct p;
    OrthOuter o;                 // kOrthLast
    int total;                   // tiles of all matrices
    uint32_t *status;
};
// E: type of the output (kOrthLast).
template <int kKind, typename E>
__global__ void __launch_bounds__(kOrthThreads, 1)
orth_pair_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb, const __grid_constant__ CUtensorMap out,
                 const __grid_constant__ CUtensorMap out_t, const OrthPairArgs a) {
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag;
    OrthPipe q = orth_pipe<2>(raw, &tmem_slot, &abort_flag);
    const int warp = ptx::warp_index();
    const OrthShare w{(int)(blockIdx.x >> 1), (int)(gridDim.x >> 1), a.total, 0, 0, (a.p.K + 63) / 64};
    ptx::grid_launch();
    ptx::grid_wait();
    // Registers of the launch, 384 x 168, as 128 x 40 (the loading and the issuing warp, two that idle) and 256 x 232: the result warps' hold their
    // 128 sums.
    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        orth_load<2>(q, a.p, w, kKind, &ta, &tb);
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if ((blockIdx.x & 1) == 0) orth_issue<2>(q, a.p, w, kKind);
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        orth_results_of<2, E>(q, a.p, w, a.o, kKind, &out, &out_t);
    }
    __syncwarp();
    orth_pipe_end<2>(q, a.status);
}

// ---- matrices in between: all products in one cooperative launch, a team of blocks to a matrix
//
// A launch per product costs some 8 us beside its work (138 us for 130 x 130, whose products take 20).  Here the blocks stay, one an SM, and
// the blocks of a team wait for one another between products: a counter in memory, some 2 us, or, where a cluster is team enough, its barrier.  Tiles are
// 128 x 128 (a cluster's also 128 x 64), a block each; where a product has fewer tiles than the team blocks, ks blocks share a tile's K: each leaves
// its sums in memory (they stay in L2), and when all of a tile's have arrived, each finishes its part of the tile's columns.  Bound by how 15 products
// follow one another: 1003 x 2601 takes 276 us, 17 us a product, of which a third multiplies (the tensor pipe is 27 % busy), the rest stores and joins
// partial sums (10000 cycles) and waits for the team (5500); 256 x 256 in a cluster 82 us.
struct OrthTeam {
    OrthOuter o;
    OrthProduct product[4];      // of each kind
    int ks[4];                   // blocks that share a tile's K
    __half *mem[4];              // X (two copies in turn), A, B
    float *part;                 // [blocks][128 columns][128 rows]
    uint32_t *counters;          // [teams] barriers, then [3][blocks] of tiles that several blocks share; zero at the start
    uint32_t *status;
    long ld_x, ld_s;
    int S, L, count, steps;
    int team, teams;             // blocks of a team, teams
};

struct OrthMaps { HalfMaps m[4]; };   // of mem

// Waits (up to two seconds, or until some block has given up) for a counter to reach `target`.  One thread.
__device__ __forceinline__ bool wait_count(const uint32_t *counter, uint32_t target, uint32_t *status, uint64_t budget_ns = ptx::kWaitBudgetNs) {
    const uint64_t t0 = ptx::globaltimer_ns();
    for (uint32_t spins = 1;; ++spins) {
        uint32_t v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
        if (v >= target) return true;
        if ((spins & 63u) == 0) {
            asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(status) : "memory");
            if (v != 0) return false;
            if (ptx::globaltimer_ns() - t0 > budget_ns) {
                atomicExch(status, 105u);
                return false;
            }
        }
    }
}
__device__ __forceinline__ void add_count(uint32_t *counter) { asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory"); }

// All blocks of the team have got here, and what they stored is seen by all.  All threads of the block; the same in all of
// them: false if some wait has given up.
__device__ __forceinline__ bool team_meet(uint32_t *counter, int members, volatile uint32_t *abort_flag, uint32_t *status, uint32_t &target,
                                          uint64_t budget_ns = ptx::kWaitBudgetNs) {
    target += members;
    const bool sound = __syncthreads_and(*abort_flag == 0) != 0;
    bool ok = true;
    if (threadIdx.x == 0) {                                  // (one thread's release and acquire cover what the barriers around them order)
        if (!sound) atomicExch(status, *abort_flag);
        add_count(counter);
        ok = wait_count(counter, target, status, budget_ns) && sound;
    }
    return __syncthreads_and(ok) != 0;
}
// The eight result warps at one barrier: whether all of them have their sums, the same in all of their threads.  A warp whose wait gave up comes here
// too: the others, whose phase may have ended in that very moment, would wait for it without a limit.
__device__ __forceinline__ bool results_agree(bool ok) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"((uint32_t)ok) : "memory");
    return all != 0;
}

// The result warps' part where ks blocks share a tile's K, once this block's sums are in memory: when all of the tile's are, its share of the tile's
// columns, eight at a time.
template <typename E>
__device__ __forceinline__ void team_join(const OrthTeam &p, const OrthPipe &q, const OrthProduct &d, const OrthTile &x, int kind, int team, int tile, int rank, int count,
                                          int ks, __half *dst) {
    const bool symmetric = orth_symmetric(kind);
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31, quad = warp & 3, half = (warp - 4) >> 2, lr = quad * 32 + lane, mat = x.mat;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (threadIdx.x == 128) {
        uint32_t *counter = p.counters + p.teams + (kind == kOrthGram ? 0 : kind == kOrthPoly ? 1 : 2) * gridDim.x + team * p.team + tile;
        add_count(counter);
        if (!wait_count(counter, (uint32_t)(ks * count), p.status)) *q.abort_flag = 106;
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const int row = x.i * 128 + lr;
    const float *all = p.part + (size_t)(team * p.team + tile * ks) * 128 * 128 + lr;
    const bool mirror = d.upper && x.i != x.j;
    if (*q.abort_flag == 0 && row < d.S) {
#pragma unroll 1
        for (int c = (rank * 2 + half) * 8; c < 128; c += 16 * ks) {
            const int col = x.j * 128 + c;
            if (col >= d.N) break;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int r = 0; r < ks; ++r) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += __ldcg(all + ((size_t)r * 128 + c + k) * 128);
            }
            if (kind == kOrthLast) {
                const OrthOuter &o = p.o;
                const size_t apart = o.tall ? (size_t)o.ld_out : 1, at = mat * o.step_out + (o.tall ? (size_t)col * o.ld_out + row : (size_t)row * o.ld_out + col);
                const int n = min(8, d.N - col);
                float old[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) old[k] = o.w && k < n ? to_f32(static_cast<const E *>(o.w)[at + k * apart]) : 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < n) from_f32(static_cast<E *>(o.out)[at + k * apart], o.w ? fmaf(-o.rate * d.f, v[k], o.keep * old[k]) : d.f * v[k]);
                continue;
            }
            const long ld = symmetric ? p.ld_s : p.ld_x, plane = (long)d.S * ld;
            __half *hi = dst + 2 * mat * plane, *lo = hi + plane;
            if (kind == kOrthPoly) {
                const __half *ah = d.a + 2 * mat * plane + (long)row * ld + col;
                float a[8];
                join8(__ldcg(reinterpret_cast<const uint4 *>(ah)), __ldcg(reinterpret_cast<const uint4 *>(ah + plane)), a);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = fmaf(d.fa, a[k], d.f * v[k]) + (row == col + k ? d.fi : 0.f);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= d.f;
            }
            uint4 vh, vl;                                            // (ld is a multiple of 8: what is beyond the last column is never read)
            split8(v, vh, vl);
            *reinterpret_cast<uint4 *>(hi + (long)row * ld + col) = vh;
            *reinterpret_cast<uint4 *>(lo + (long)row * ld + col) = vl;
            if (mirror) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (col + k < d.N) split_half(v[k], hi[(long)(col + k) * ld + row], lo[(long)(col + k) * ld + row]);
            }
        }
    }
    asm volatile("fence.proxy.async.global;" ::: "memory");              // (loaded by TMA next)
    __syncwarp();
}
template <bool kCluster, bool kResults, typename E>
__device__ __forceinline__ void team_product(const OrthTeam &p, OrthPipe &q, int kind, int team, int mat, int count, const HalfMaps *ta, const HalfMaps *tb,
                                             const HalfMaps *out, __half *dst) {
    const bool symmetric = orth_symmetric(kind);
    const int warp = ptx::warp_index(), member = blockIdx.x % p.team;
    const OrthProduct &d = p.product[kind];
    const int blocks = (d.K + 63) / 64, ks = kCluster ? 1 : p.ks[kind];
    // (with ks blocks a tile: member ks t + r has the r-th part of tile t's K, and no second tile)
    const int rank = ks > 1 ? member % ks : 0, first = member / ks;
    if (ks > 1 && first >= d.tiles) return;
    const OrthShare w{first, ks > 1 ? d.tiles : p.team, d.tiles, mat, blocks * rank / ks, blocks * (rank + 1) / ks};
    if constexpr (!kResults) {
        if (warp == 0) orth_load<1>(q, d, w, kind, &ta->load, &tb->load);
        else if (warp == 1) orth_issue<1>(q, d, w, kind);
    } else {
        const int quad = warp & 3, half = (warp - 4) >> 2, lane = threadIdx.x & 31, chunks = (w.kb1 - w.kb0 + orth_chunk(kind) - 1) / orth_chunk(kind);
        for (int t = w.t0; t < w.total; t += w.step) {
            const OrthTile x = orth_tile(d, w, t);
            float v[64];
            const bool mine = half * 64 < d.width;
            const int row0 = x.i * 128 + quad * 32, col0 = mine ? x.j * d.width + half * 64 : d.N;
            const bool only = (kCluster || ks == 1) && d.tiles <= p.team;    // (this block's one tile)
            bool ok = orth_sums<1>(q, chunks, v, mine);
            if (only) ok = results_agree(ok);                                // (everybody's sums are complete, so no stage is in use)
            if (!ok) break;
            if (kCluster || ks == 1) {
                const bool mirror = d.upper && x.i != x.j;
                if (only) {
                    orth_finish<true, E>(q, d, p.o, kind, mat, row0, col0, mirror, &out->store, &out->store_t, v);
                } else {
                    orth_finish<false, E>(q, d, p.o, kind, mat, row0, col0, mirror, &out->store, &out->store_t, v);
                }
            } else {
                float *mine = p.part + (size_t)blockIdx.x * 128 * 128 + (half * 64) * 128 + quad * 32 + lane;
#pragma unroll
                for (int k = 0; k < 64; ++k) __stcg(mine + k * 128, v[k]);
            }
        }
        if (!kCluster && ks > 1) team_join<E>(p, q, d, orth_tile(d, w, first), kind, team, first, rank, count, ks, dst);
        else if (lane == 0) ptx::tma_store_wait<false>();
        asm volatile("fence.proxy.async.global;" ::: "memory");
        __syncwarp();
    }
    __syncwarp();
}

template <bool kCluster, bool kResults, typename E>
__device__ __forceinline__ void team_run(const OrthMaps &maps, const OrthTeam &p, OrthPipe &q) {
    const int team = blockIdx.x / p.team;
    uint32_t met = 0;
    bool ok = true;
    int count = 0;                                           // steps this team has begun
    for (int mat = team; mat < p.count && (kCluster || ok); mat += p.teams)
        // three products a step, one piece of code for all
        for (int i = 0; i < 3 * p.steps && (kCluster || ok); ++i) {
            const int step = i / 3, stage = i - 3 * step, cur = step & 1, kind = stage < 2 ? stage : step + 1 < p.steps ? kOrthApply : kOrthLast;
            const int left = stage == 0 ? cur : stage == 1 ? 2 : 3, right = stage == 1 ? 2 : cur, to = stage == 0 ? 2 : stage == 1 ? 3 : 1 - cur;
            count += stage == 0;
            if (ok) team_product<kCluster, kResults, E>(p, q, kind, team, mat, count, maps.m + left, maps.m + right, maps.m + to, p.mem[to]);
            if constexpr (kCluster) {
                // (a block that gave up a wait, as a whole, does no further product, for its roles are no longer at the same stage, but meets the others)
                ok = __syncthreads_and(ok && *q.abort_flag == 0) != 0;
                ptx::cluster_meet();
            } else if (kind != kOrthLast || mat + p.teams < p.count) {
                ok = team_meet(p.counters + team, p.team, q.abort_flag, p.status, met);
            }
        }
}
// kCluster: the team is a cluster, whose barrier takes a tenth of the time; else a cooperative launch.
template <bool kCluster, typename E>
__global__ void __launch_bounds__(kOrthThreads, 1) orth_team_kernel(const __grid_constant__ OrthMaps maps, const __grid_constant__ OrthTeam p) {
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag;
    OrthPipe q = orth_pipe<1>(raw, &tmem_slot, &abort_flag);
    ptx::grid_launch();
    ptx::grid_wait();
    // Registers of the launch, 384 x 168, as 128 x 72 and 256 x 216.
    if (ptx::warp_index() < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        team_run<kCluster, false, E>(maps, p, q);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        team_run<kCluster, true, E>(maps, p, q);
    }
    __syncwarp();
    orth_pipe_end<1>(q, p.status);
}

// How a team ends when its waits run out, on its own: two blocks as the team kernel has them, at the end of two products, of which in the first block one
// result warp is said to have given up (gone = 1), or which wait for a third that is not there (gone = 2).  out: [2][12 warps], bit 0 that the warp
// went on after results_agree (the first four warps: always), bit 1 that it went on after both meetings; then [2] nanoseconds that what is in flight was given.
__global__ void __launch_bounds__(kOrthThreads, 1) selftest_team_kernel(uint32_t *status, uint32_t *counter, uint32_t *out, int gone, uint64_t budget_ns) {
    __shared__ volatile uint32_t abort_flag;
    if (threadIdx.x == 0) abort_flag = 0;
    __syncthreads();
    const int warp = ptx::warp_index();
    bool agreed = true;
    if (warp >= 4) {
        const bool lost = gone == 1 && blockIdx.x == 0 && warp == 7;
        if (lost && (threadIdx.x & 31) == 0) abort_flag = 104;
        __syncwarp();
        agreed = results_agree(!lost);
    }
    uint32_t target = 0;
    bool met = true;
    for (int i = 0; i < 2 && met; ++i) met = team_meet(counter, gone == 2 ? 3 : 2, &abort_flag, status, target, budget_ns);
    const uint64_t t0 = ptx::globaltimer_ns();
    let_arrive(&abort_flag);
    if (threadIdx.x == 0) out[24 + blockIdx.x] = (uint32_t)(ptx::globaltimer_ns() - t0);
    if ((threadIdx.x & 31) == 0) out[blockIdx.x * 12 + warp] = (agreed ? 1u : 0u) | (met ? 2u : 0u);
}

// ---------------------------------------------------------------- a whole matrix in one block
// S up to 128 and everything in shared memory: X as panels of 64 columns, rows of 128 bytes (128-byte swizzle), Mr = S rounded up to 16 of them in high
// halves and below them as many in low ones, and behind them A, overwritten by B, in the same form.  The same bytes serve as rows of X
// (sums along rows) and as the right factor of B X (sums over rows).  The MMAs have 128 rows whatever S is; what they read beyond a panel's
// rows is what lies behind it, and its sums are not looked at.  Bound by how long the parts of a step follow one another: the MMAs read their
// factors from shared memory (8 of 256 x 16 take 19 us, 24 of 128 x 128 39 us, whatever else runs beside them; 128 x 128 x 16: 95 cycles for 64 of arithmetic; as here with high and low rows side by side 110 for two of them), and every
// sum goes through tensor memory, registers and a split once a product.
//
// kNarrow (S up to 64): one MMA forms high high, high low and low high of X X^T at a time (rows and columns of both halves; the third part comes over from
// the lanes below), and B X is formed as its transpose, columns of X on the 128 lanes, which all have work then.  A step at 16 x 256: 5400
// cycles, 7100 without.
struct OrthSmall {
    OrthOuter o;
    OrthScales sc;
    int S, L, Mr, panels, steps;
    uint32_t *status;
};
constexpr int kOrthSmallThreads = 512;
struct OrthSmallSize {
    size_t x, a, scratch, total;                                    // bytes of X and of A; where the scratch is, and the end
};
__host__ __device__ inline OrthSmallSize orth_small_size(int S, int L) {
    OrthSmallSize z;
    const size_t Mr = (size_t)(S + 15) / 16 * 16;
    z.x = (size_t)((L + 63) / 64) * 2 * Mr * 128;
    z.a = (size_t)((S + 63) / 64) * 2 * Mr * 128;
    // what an MMA reads beyond the last panel is there: 128 rows from its first high row on (S up to 64), from its first low row on (above)
    const size_t rows = S <= 64 ? 2 * Mr : Mr;
    z.scratch = 1024 + z.x + z.a + (rows < 128 ? (128 - rows) * 128 : 0);
    z.total = z.scratch + (S <= 64 ? Mr * Mr * sizeof(float) : 0) + 64;
    return z;
}
// Byte offset of the eight columns from c (a multiple of 8) on of a row, `rows` rows a panel.
__device__ __forceinline__ uint32_t panel_at(int row, int c, int rows) { return (uint32_t)((c >> 6) * rows + row) * 128 + ((((uint32_t)c >> 3) & 7) ^ (row & 7)) * 16; }

template <bool kNarrow>
__global__ void __launch_bounds__(kOrthSmallThreads, 1) orth_small_kernel(const OrthSmall p) {
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag;
    __shared__ __align__(8) uint64_t bar_word;
    __shared__ double sums[kOrthSmallThreads / 32];
    uint8_t *smem = ptx::align_1024(raw);
    const OrthSmallSize z = orth_small_size(p.S, p.L);
    const int Mr = p.Mr, Pr = 2 * Mr;                                // rows of a half, of a panel
    const uint32_t low = (uint32_t)Mr * 128, panel = (uint32_t)Pr * 128;   // bytes from a high row to its low one, of a panel
    uint8_t *xs = smem, *as = smem + z.x;
    const uint32_t bar = ptx::smem_u32(&bar_word);
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
    const size_t mat = blockIdx.x;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        ptx::mbar_init(bar, 1);
        ptx::fence_mbar_init();
    }
    if (warp == 0) ptx::tmem_alloc(ptx::smem_u32(&tmem_slot), 512);
    // zeros in the rows and columns that X and A do not fill (and everywhere else, once)
    for (size_t i = threadIdx.x; i < (z.scratch - 1024) / 16; i += kOrthSmallThreads) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    ptx::grid_launch();
    ptx::grid_wait();
    const OrthOuter &o = p.o;
    if (o.w) {                                                       // (the weights are wanted at the end)
        const size_t e = o.out_type == 0 ? 4 : 2, bytes = (size_t)o.rows * o.cols * e;
        for (size_t at = (size_t)threadIdx.x * 128; at < bytes; at += kOrthSmallThreads * 128)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const char *>(o.w) + mat * o.step_out * e + at));
    }
    // the elements once from memory: as float32, its two 16-bit parts where the halves will be, and their squares
    double sum = 0.0;
    orth_elements<false>(o, mat, threadIdx.x, kOrthSmallThreads, [&](int r, int c, const auto &u) {
        constexpr int V = sizeof(u) / sizeof(float);
        for (float x : u) sum += (double)x * x;
        if (V == 4 && !o.tall) {
            uint32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(u[i % V]);
            uint8_t *at = xs + panel_at(r, c & ~7, Pr) + (c & 7) * 2;
            *reinterpret_cast<uint2 *>(at) = make_uint2(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632));
            *reinterpret_cast<uint2 *>(at + low) = make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int s = o.tall ? c + i : r, l = o.tall ? r : c + i;
                uint8_t *at = xs + panel_at(s, l & ~7, Pr) + (l & 7) * 2;
                const uint32_t b = __float_as_uint(u[i]);
                *reinterpret_cast<uint16_t *>(at) = (uint16_t)(b >> 16);
                *reinterpret_cast<uint16_t *>(at + low) = (uint16_t)b;
            }
        }
    });
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < kOrthSmallThreads / 32; ++k) sum += sums[k];
    const double f = (double)p.sc.x / (sqrt(sum) + (double)o.eps);
    for (int i = threadIdx.x; i < p.panels * Mr * 8; i += kOrthSmallThreads) {
        uint8_t *at = xs + (uint32_t)(i / (8 * Mr)) * panel + (uint32_t)(i % (8 * Mr)) * 16;
        const uint4 h = *reinterpret_cast<const uint4 *>(at), l = *reinterpret_cast<const uint4 *>(at + low);
        const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = (float)(__uint_as_float(__byte_perm(hw[k], lw[k], 0x1054)) * f);
            v[2 * k + 1] = (float)(__uint_as_float(__byte_perm(hw[k], lw[k], 0x3276)) * f);
        }
        uint4 vh, vl;
        split8(v, vh, vl);
        *reinterpret_cast<uint4 *>(at) = vh;
        *reinterpret_cast<uint4 *>(at + low) = vl;
    }
    ptx::fence_proxy_async_smem();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = tmem_slot;

    uint32_t phase = 0;
    constexpr uint32_t hi = ptx::desc_hi(1024, 2);
    constexpr int kParts = kOrthSmallThreads / 128, kTurns = kNarrow ? 1 : 2;   // warps that share a quarter of the lanes; sixteen columns a turn of theirs cover Mr
    const uint32_t dx = ptx::smem_u32(xs), da = ptx::smem_u32(as);
    const int quad = warp & 3, part = warp >> 2, row = quad * 32 + lane, deep_s = Mr / 16, deep_l = (p.L + 15) / 16;
    const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16);
    const float fg = p.sc.a / (p.sc.x * p.sc.x), fp = p.sc.cc * p.sc.b / (p.sc.a * p.sc.a), fa = p.sc.cb * p.sc.b / p.sc.a, fi = p.sc.ca * p.sc.b, fx = 1.f / p.sc.b;
    float *scratch = reinterpret_cast<float *>(smem + z.scratch - 1024);        // [column][row]: low high, on its way to the lanes of the high rows
    auto mma = [&](uint32_t d, uint32_t a, uint32_t a_lbo, uint32_t b, uint32_t b_lbo, uint32_t idesc, bool more) {
        ptx::mma_ss(d, ptx::desc(ptx::desc_lo(a, a_lbo), hi), ptx::desc(ptx::desc_lo(b, b_lbo), hi), idesc, more);
    };
    auto finish = [&]() {
        // (every thread waits; whether to go on is agreed on by all)
        const bool ok = ptx::mbar_wait(bar, phase, &abort_flag, 111);
        phase ^= 1;
        ptx::tc_fence_after();
        return __syncthreads_and(ok) != 0;
    };
    auto ready = [&]() {
        ptx::fence_proxy_async_smem();
        ptx::tc_fence_before();
        __syncthreads();
        ptx::tc_fence_after();
    };
    // High rows times high and low rows (columns 0.. and Mr.. of the sums), and low rows times high ones (narrow: rows Mr.. of the sums, else added to the
    // first), of the panels from `at` on, `deep` times sixteen columns.
    auto square = [&](uint32_t at, int deep) {
        if (warp == 0 && ptx::elect_one()) {
            const uint32_t both = instr_desc_f16(128, 2 * Mr, 0), one = instr_desc_f16(128, Mr, 0);
            for (int k = 0; k < deep; ++k) {
                const uint32_t c = at + (k >> 2) * panel + (k & 3) * 32;
                mma(tmem, c, 16, c, 16, both, k > 0);
                if (!kNarrow) mma(tmem, c + low, 16, c, 16, one, true);
            }
            ptx::mma_commit(bar);
        }
        __syncwarp();
    };
    // its parts added up, sixteen columns at a time of the rows below Mr: use(turn, column, sums)
    auto sums_of = [&](auto use) {
        if constexpr (kNarrow) {
            if (part * 16 < Mr) {
                uint32_t u[16];
                ptx::tmem_ld16(acc + part * 16, u);
                ptx::tmem_wait_ld();
                if (row >= Mr && row < 2 * Mr) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) scratch[(part * 16 + k) * Mr + row - Mr] = __uint_as_float(u[k]);
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < kTurns; ++j) {
            const int c = (part + j * kParts) * 16;
            if (quad * 32 >= Mr || c >= Mr) continue;                           // (uniform over the warp)
            uint32_t u[16], w[16];
            ptx::tmem_ld16(acc + c, u);
            ptx::tmem_ld16(acc + Mr + c, w);
            ptx::tmem_wait_ld();
            if (row < Mr) {
                float v[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = (kNarrow ? __uint_as_float(w[k]) + scratch[(c + k) * Mr + row] : __uint_as_float(w[k])) + __uint_as_float(u[k]);
                use(j, c, v);
            }
            __syncwarp();
        }
    };
    auto store16 = [&](uint8_t *to, int c, const float *v) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint4 vh, vl;
            split8(v + 8 * q, vh, vl);
            uint8_t *at = to + panel_at(row, c + 8 * q, Pr);
            *reinterpret_cast<uint4 *>(at) = vh;
            *reinterpret_cast<uint4 *>(at + low) = vl;
        }
    };
    float keep[kTurns][16];                                                     // this thread's part of A
    bool ok = true;
    for (int step = 0; step < p.steps && ok; ++step) {
        // A = X X^T
        square(dx, deep_l);
        if (!(ok = finish())) break;
        sums_of([&](int j, int c, float (&v)[16]) {
#pragma unroll
            for (int k = 0; k < 16; ++k) keep[j][k] = v[k] *= fg;
            store16(as, c, v);
        });
        ready();
        // B = a I + b A + c A^2, over A
        square(da, deep_s);
        if (!(ok = finish())) break;
        sums_of([&](int j, int c, float (&v)[16]) {
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = fmaf(fa, keep[j][k], fp * v[k]) + (row == c + k ? fi : 0.f);
            store16(as, c, v);
        });
        ready();
        if constexpr (kNarrow) {
            // X^T <- X^T B: 128 columns of X a group, 2 Mr columns of sums each, as many groups at a time as tensor memory holds
            const int groups = (p.L + 127) / 128, at_once = 256 / Mr, pieces = Mr / 16;
            for (int g0 = 0; g0 < groups; g0 += at_once) {
                const int g1 = min(g0 + at_once, groups);
                if (warp == 0 && ptx::elect_one()) {
                    const uint32_t across = 1u << 15;                           // (the left factor's columns are the ones next to each other)
                    const uint32_t both = instr_desc_f16(128, 2 * Mr, 0) | across, one = instr_desc_f16(128, Mr, 0) | across;
                    for (int g = g0; g < g1; ++g)
                        for (int k = 0; k < deep_s; ++k) {
                            const uint32_t d = tmem + (g - g0) * 2 * Mr, x = dx + 2 * g * panel + k * 2048, b = da + k * 32;
                            mma(d, x, panel, b, 16, both, k > 0);
                            mma(d, x + low, panel, b, 16, one, true);
                        }
                    ptx::mma_commit(bar);
                }
                __syncwarp();
                if (!(ok = finish())) break;
                for (int i = part; i < (g1 - g0) * pieces; i += kParts) {       // sixteen rows of X of a group
                    const int g = i / pieces, c = i % pieces * 16, l = (g0 + g) * 128 + row;
                    uint32_t u[16], w[16];
                    ptx::tmem_ld16(acc + g * 2 * Mr + c, u);
                    ptx::tmem_ld16(acc + g * 2 * Mr + Mr + c, w);
                    ptx::tmem_wait_ld();
                    if (l < 64 * p.panels) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            uint8_t *at = xs + panel_at(c + k, l & ~7, Pr) + (l & 7) * 2;
                            split_half(fx * (__uint_as_float(u[k]) + __uint_as_float(w[k])), *reinterpret_cast<__half *>(at), *reinterpret_cast<__half *>(at + low));
                        }
                    }
                    __syncwarp();
                }
                ready();
            }
        } else {
            // X <- B X, as many columns at a time as tensor memory holds
            for (int l0 = 0; l0 < 64 * p.panels; l0 += 512) {
                const int l1 = min(l0 + 512, 64 * p.panels);
                if (warp == 0 && ptx::elect_one()) {
                    for (int l = l0; l < l1; l += 256) {
                        const uint32_t idesc = instr_desc_f16(128, min(256, l1 - l), 1);
                        for (int k = 0; k < deep_s; ++k) {
                            const uint32_t d = tmem + (l - l0), b = da + (k >> 2) * panel + (k & 3) * 32, x = dx + (l >> 6) * panel + k * 2048;
                            mma(d, b + low, 16, x, panel, idesc, k > 0);
                            mma(d, b, 16, x + low, panel, idesc, true);
                            mma(d, b, 16, x, panel, idesc, true);
                        }
                    }
                    ptx::mma_commit(bar);
                }
                __syncwarp();
                if (!(ok = finish())) break;
                for (int l = l0 + part * 16; l < l1; l += 16 * kParts) {
                    uint32_t u[16];
                    ptx::tmem_ld16(acc + (l - l0), u);
                    ptx::tmem_wait_ld();
                    if (row < Mr) {
                        float v[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(u[k]) * fx;
                        store16(xs, l, v);
                    }
                    __syncwarp();
                }
                ready();
            }
        }
    }
    // the result, from its halves
    const float back = 1.f / p.sc.x;
    orth_results(o, mat, threadIdx.x, kOrthSmallThreads, [&](int r, int c, auto &v) {
        constexpr int V = sizeof(v) / sizeof(float);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int s = o.tall ? c + i : r, l = o.tall ? r : c + i;
            const uint8_t *at = xs + panel_at(s, l & ~7, Pr) + (l & 7) * 2;
            v[i] = back * (__half2float(*reinterpret_cast<const __half *>(at)) + __half2float(*reinterpret_cast<const __half *>(at + low)));
        }
    });
    ptx::tc_fence_before();
    __syncthreads();
    let_arrive(&abort_flag);
    if (threadIdx.x == 0 && abort_flag != 0) p.status[0] = abort_flag;
    if (warp == 0) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace flare
