// Orthogonalising an update by Newton-Schulz products:  X0 = U / (|U|_F + eps),  then `steps` times
//
//     A = X X^T,   B = a I + b A + c A^2,   X <- B X                      (the odd quintic a x + b x^3 + c x^5 of the singular values)
//
// with X [S, L], S the short side (U transposed where it is tall).  The quintic lifts small singular values by up to a^steps (485 for
// the usual coefficients), and with them whatever was rounded away of X beside its large ones: bfloat16 or tf32 factors (8, 11 bits)
// are off by several percent after five steps on matrices with a few strong directions.  So every factor is carried as two float16
// halves (22 bits), x = hi + lo at a power-of-two scale that keeps lo a normal number, and a product is hi hi + hi lo + lo hi on the
// tensor cores with float32 sums: three products at the 16-bit rate against one at a rate some twenty times lower in float32.
// A, B and the squares are symmetric: only tiles on and above the diagonal are computed, each is stored twice.
#pragma once

#include "flare_common.cuh"
#include "flare_ptx.cuh"

namespace flare {

// What a step's products are for.
enum { kOrthGram = 0, kOrthPoly = 1, kOrthApply = 2, kOrthLast = 3 };

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

// ---------------------------------------------------------------- norm and first split, for matrices that do not fit a block
constexpr int kOrthNormThreads = 256;

// Momentum, and per block the sum of squares of its share of a matrix, in float64 (gradients of 1e-25 are as good as any).  Grid (blocks, count).
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
// The halves of X0, [2 count][S][ld] (high and low of a matrix in turn).  Rows as they lie: grid (blocks, 1, count).  tall: tiles of 64 x 64 through
// shared memory, grid (col tiles, row tiles, count).
__global__ void __launch_bounds__(256) orth_split_kernel(OrthOuter o, const double *part, int parts, __half *x, long ld, float scale) {
    __shared__ float tile[64][65];
    __shared__ double norm_sh;
    ptx::grid_launch();
    ptx::grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const size_t mat = blockIdx.z;
    if (warp == 0) {
        double sum = 0.0;
        for (int i = lane; i < parts; i += 32) sum += part[mat * parts + i];
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        if (lane == 0) norm_sh = (double)scale / (sqrt(sum) + (double)o.eps);
    }
    const int S = o.tall ? o.cols : o.rows, L = o.tall ? o.rows : o.cols;
    __half *hi = x + 2 * mat * S * ld, *lo = hi + S * ld;
    if (!o.tall) {
        __syncthreads();
        const double f = norm_sh;
        orth_elements<true>(o, mat, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256, [&](int r, int c, const auto &u) {
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
    // the tile as a matrix of its own
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    with_type(o.g_type, [&](auto type) {
        using G = decltype(type);
        const G *g = static_cast<const G *>(o.g) + mat * o.step_g;
        const float *m = o.m ? o.m_out + mat * (size_t)o.rows * o.cols : nullptr;
#pragma unroll
        for (int i0 = 0; i0 < 16; i0 += 8) {
            float u[8], q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = r0 + (i0 + i) * 4 + (threadIdx.x >> 6), c = c0 + (threadIdx.x & 63);
                const bool yes = r < o.rows && c < o.cols;
                u[i] = yes ? to_f32(g[(size_t)r * o.ld_g + c]) : 0.f;
                q[i] = yes && m ? m[(size_t)r * o.cols + c] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                tile[(i0 + i) * 4 + (threadIdx.x >> 6)][threadIdx.x & 63] = !m ? u[i] : o.nesterov ? fmaf(o.momentum, q[i], (1.f - o.momentum) * u[i]) : q[i];
        }
    });
    __syncthreads();
    const double f = norm_sh;
    const int l = r0 + 2 * lane;
    for (int s = warp; s < 64; s += 8)
        if (c0 + s < S && l < L) {                                   // (ld is even; what is beyond the last column is never read)
            uint32_t low;
            const uint32_t high = half_pair((float)(tile[2 * lane][s] * f), (float)(tile[2 * lane + 1][s] * f), low);
            const size_t at = (size_t)(c0 + s) * ld + l;
            *reinterpret_cast<uint32_t *>(hi + at) = high;
            *reinterpret_cast<uint32_t *>(lo + at) = low;
        }
}

// ---------------------------------------------------------------- one product
// Instruction descriptor for kind::f16 with float16 operands and float accumulation.
__host__ __device__ constexpr uint32_t instr_desc_f16(int m, int n, int b_mn) {
    return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

struct OrthProduct {
    __half *dst;                 // halves of the result [2 count][S][ld_dst]
    const __half *a;             // halves of A (kOrthPoly) [2 count][S][ld_a]
    long ld_dst, ld_a;
    int S, N, K;                 // result [S, N], sums over K
    int tiles_m, tiles_n, tiles; // tiles of a matrix, down, across and in all
    int total;                   // of all matrices
    int ks;                      // blocks of a cluster that share a tile's K (single blocks only)
    float f, fa, fi;             // result = f sums (+ fa A + fi I)
    OrthOuter o;                 // kOrthLast
    uint32_t *status;
};

// Warp 0 loads, warp 1 issues, warps 4 to 11 take the sums out of tensor memory.
constexpr int kOrthThreads = 384, kOrthStages = 3, kOrthChunk = 8;  // 64-deep steps whose sums stay in tensor memory
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

// E: type of the output (kOrthLast).
template <int kKind, int kPair, typename E>
__global__ void __launch_bounds__(kOrthThreads, 1)
orth_product_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb, const __grid_constant__ CUtensorMap out,
                    const __grid_constant__ CUtensorMap out_t, const OrthProduct p) {
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag;
    uint8_t *smem = ptx::align_1024(raw);
    constexpr bool kSymmetric = kKind == kOrthGram || kKind == kOrthPoly;
    constexpr int kTileN = 128 * kPair, kCols = kTileN / 2;              // columns of the tile, of a result warp
    const uint32_t smem0 = ptx::smem_u32(smem), pieces0 = smem0 + kOrthStages * kOrthStage, bars = pieces0 + 8 * kOrthPiece;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (kOrthStages + s); };
    auto acc_full = [&](int b) { return bars + 8 * (2 * kOrthStages + b); };
    auto acc_empty = [&](int b) { return bars + 8 * (2 * kOrthStages + 2 + b); };
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
    const int in_pair = kPair == 2 ? (int)(blockIdx.x & 1) : 0;          // this block's half of the pair's tile
    const int rank = kPair == 1 && p.ks > 1 ? (int)(blockIdx.x % p.ks) : 0, group = blockIdx.x / (kPair * p.ks), groups = gridDim.x / (kPair * p.ks);
    const int blocks = (p.K + 63) / 64, kb0 = (int)((long)blocks * rank / p.ks), kb1 = (int)((long)blocks * (rank + 1) / p.ks);
    const int chunks = (kb1 - kb0 + kOrthChunk - 1) / kOrthChunk;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int s = 0; s < kOrthStages; ++s) { ptx::mbar_init(full(s), 1); ptx::mbar_init(empty(s), 1); }
        for (int b = 0; b < 2; ++b) { ptx::mbar_init(acc_full(b), 1); ptx::mbar_init(acc_empty(b), 8 * kPair); }
        ptx::fence_mbar_init();
    }
    if (warp == 1) ptx::tmem_alloc_for<kPair>(ptx::smem_u32(&tmem_slot), 2 * kTileN);
    ptx::tc_fence_before();
    __syncthreads();
    if (kPair == 2) ptx::cluster_meet();
    ptx::tc_fence_after();
    const uint32_t tmem = tmem_slot;
    ptx::grid_launch();
    ptx::grid_wait();

    struct Tile { int mat, i, j; };
    auto tile_of = [&](int t) {
        Tile x;
        x.mat = t / p.tiles;
        t -= x.mat * p.tiles;
        if (kSymmetric) upper_tile(t, p.tiles_n, x.i, x.j);
        else { x.i = t % p.tiles_m; x.j = t / p.tiles_m; }
        return x;
    };
    // Registers of a pair's launch, 384 x 168, as 128 x 40 (this and the issuing warp, two that idle) and 256 x 232: the result warps' hold their
    // 128 sums.
    if (warp == 0) {
        if (kPair == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (ptx::elect_one()) {
            asm volatile("fence.proxy.async.global;" ::: "memory");      // (what the launches before this one stored, for the loads by TMA)
            uint32_t n = 0;
            bool ok = true;
            for (int t = group; t < p.total && ok; t += groups) {
                const Tile x = tile_of(t);
                const bool own = kSymmetric && x.i == x.j;               // both factors are the same rows
                const int ra = x.i * kTileN + in_pair * 128, rb = x.j * kTileN + in_pair * 128;
                for (int kb = kb0; kb < kb1; ++kb, ++n) {
                    const int s = n % kOrthStages;
                    if (n >= kOrthStages && !(ok = ptx::mbar_wait(empty(s), (n / kOrthStages - 1) & 1, &abort_flag, 101))) break;
                    const uint32_t at = smem0 + s * kOrthStage, bar = kPair == 2 ? ptx::in_block(full(s), 0) : full(s);
                    if (in_pair == 0) ptx::mbar_arrive_expect_tx(full(s), kPair * (own ? 2 : 4) * kOrthHalfTile);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            ptx::tma_load_3d_for<kPair>(at + h * kOrthHalfTile + q * 8192, &ta, bar, kb * 64, ra + q * 64, 2 * x.mat + h);
                            if (own) continue;
                            if (kSymmetric) ptx::tma_load_3d_for<kPair>(at + (2 + h) * kOrthHalfTile + q * 8192, &tb, bar, kb * 64, rb + q * 64, 2 * x.mat + h);
                            else ptx::tma_load_3d_for<kPair>(at + (2 + h) * kOrthHalfTile + q * 8192, &tb, bar, rb + q * 64, kb * 64, 2 * x.mat + h);
                        }
                }
            }
        }
        __syncwarp();
        if (kPair == 1 && p.ks > 1) ptx::cluster_meet();
    } else if (warp == 1) {
        if (kPair == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (in_pair == 0 && ptx::elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(128 * kPair, kTileN, kSymmetric ? 0 : 1), hi = ptx::desc_hi(1024, 2);
            constexpr uint32_t b_lbo = kSymmetric ? 16 : 8192, b_step = (kSymmetric ? 32 : 2048) >> 4, low = kOrthHalfTile >> 4;
            uint32_t n = 0, c = 0;
            bool ok = true;
            for (int t = group; t < p.total && ok; t += groups) {
                const Tile x = tile_of(t);
                const bool own = kSymmetric && x.i == x.j;
                for (int kb = kb0; kb < kb1 && ok; ++c) {
                    const uint32_t acc = tmem + (c & 1) * kTileN;
                    if (c >= 2 && !(ok = ptx::mbar_wait(acc_empty(c & 1), (c / 2 - 1) & 1, &abort_flag, 102))) break;
                    ptx::tc_fence_after();
                    for (int k1 = min(kb + kOrthChunk, kb1), first = 1; kb < k1; ++kb, ++n, first = 0) {
                        const int s = n % kOrthStages;
                        if (!(ok = ptx::mbar_wait(full(s), (n / kOrthStages) & 1, &abort_flag, 103))) break;
                        ptx::tc_fence_after();
                        const uint32_t at = smem0 + s * kOrthStage;
                        const uint32_t a0 = ptx::desc_lo(at, 16), b0 = ptx::desc_lo(own ? at : at + 2 * kOrthHalfTile, b_lbo);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t a = a0 + k * 2, b = b0 + k * b_step;
                            ptx::mma_ss_for<kPair>(acc, ptx::desc(a + low, hi), ptx::desc(b, hi), idesc, !first || k > 0);
                            ptx::mma_ss_for<kPair>(acc, ptx::desc(a, hi), ptx::desc(b + low, hi), idesc, 1);
                            ptx::mma_ss_for<kPair>(acc, ptx::desc(a, hi), ptx::desc(b, hi), idesc, 1);
                        }
                        ptx::mma_commit_for<kPair>(empty(s));
                    }
                    if (ok) ptx::mma_commit_for<kPair>(acc_full(c & 1));
                }
            }
        }
        __syncwarp();
        if (kPair == 1 && p.ks > 1) ptx::cluster_meet();
    } else if (warp < 4) {
        if (kPair == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (kPair == 1 && p.ks > 1) ptx::cluster_meet();
    } else {
        if (kPair == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int quad = warp & 3, half = (warp - 4) >> 2, lr = quad * 32 + lane;
        const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + half * kCols;
        const uint32_t piece = pieces0 + (warp - 4) * kOrthPiece;
        uint8_t *piece_p = smem + kOrthStages * kOrthStage + (warp - 4) * kOrthPiece;
        uint32_t c = 0;
        bool ok = true;
        for (int t = group; t < p.total && ok; t += groups) {
            const Tile x = tile_of(t);
            float v[kCols];
            for (int q = 0; q < chunks; ++q, ++c) {
                ok = ptx::mbar_wait(acc_full(c & 1), (c / 2) & 1, &abort_flag, 104);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                ptx::tc_fence_after();
#pragma unroll
                for (int k = 0; k < kCols; k += 32) {
                    uint32_t u[32];
                    ptx::tmem_ld32(acc + (c & 1) * kTileN + k, u);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[k + e] = q == 0 ? __uint_as_float(u[e]) : v[k + e] + __uint_as_float(u[e]);
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (kPair == 2) ptx::mbar_arrive_cluster(ptx::in_block(acc_empty(c & 1), 0));
                    else ptx::mbar_arrive(acc_empty(c & 1));
                }
            }
            if (!ok) break;
            const int row0 = x.i * kTileN + in_pair * 128 + quad * 32, row = row0 + lane, col0 = x.j * kTileN + half * kCols;
            if (kPair == 1 && p.ks > 1) {
                // the cluster's sums meet below: this block's in shared memory by columns
                float *part = reinterpret_cast<float *>(smem);
#pragma unroll
                for (int k = 0; k < kCols; ++k) part[(half * kCols + k) * 128 + lr] = v[k];
                break;
            }
            if (kKind == kOrthLast) {
#pragma unroll
                for (int k = 0; k < kCols; k += 32)
                    if (row0 < p.S && col0 + k < p.N)
                        outer_piece<E>(p.o, x.mat, row0, col0 + k, p.S, p.N, v + k, p.f, reinterpret_cast<float *>(piece_p));
                continue;
            }
            const __half *ah = p.a + 2 * x.mat * (long)p.S * p.ld_a + (long)row * p.ld_a + col0, *al = ah + (long)p.S * p.ld_a;
#pragma unroll
            for (int k = 0; k < kCols; k += 8) {
                float a[8];
                if (kKind == kOrthPoly) {
                    uint4 h = make_uint4(0, 0, 0, 0), l = h;
                    if (row < p.S && col0 + k < p.N) {
                        h = *reinterpret_cast<const uint4 *>(ah + k);
                        l = *reinterpret_cast<const uint4 *>(al + k);
                    }
                    join8(h, l, a);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[k + e] = kKind == kOrthPoly ? fmaf(p.fa, a[e], p.f * v[k + e]) + (row == col0 + k + e ? p.fi : 0.f) : p.f * v[k + e];
            }
#pragma unroll
            for (int k = 0; k < kCols; k += 64) {
                if (row0 >= p.S || col0 + k >= p.N) continue;            // (uniform over the warp)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // 32 rows of 64 columns, 128-byte swizzle; then what the other half is formed from
                    if (lane == 0) ptx::tma_store_wait<true>();
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 64; e += 8) {
                        uint4 vh, vl;
                        split8(v + k + e, vh, vl);
                        const uint4 &w = h == 0 ? vh : vl;
                        const uint32_t r[4] = {w.x, w.y, w.z, w.w};
                        ptx::sts128(piece + lane * 128 + (((e >> 3) ^ (lane & 7)) << 4), r);
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        ptx::tma_store_3d(&out, piece, col0 + k, row0, 2 * x.mat + h);
                        ptx::tma_store_commit();
                    }
                    if (!kSymmetric || x.i == x.j) continue;
                    // the same 64 columns as rows of 32: 64-byte swizzle
                    if (lane == 0) ptx::tma_store_wait<true>();
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 64; ++e) {
                        __half vh, vl;
                        split_half(v[k + e], vh, vl);
                        *reinterpret_cast<__half *>(piece_p + e * 64 + (((lane >> 3) ^ ((e >> 1) & 3)) << 4) + (lane & 7) * 2) = h == 0 ? vh : vl;
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        ptx::tma_store_3d(&out_t, piece, row0, col0 + k, 2 * x.mat + h);
                        ptx::tma_store_commit();
                    }
                }
            }
        }
        if (lane == 0) ptx::tma_store_wait<false>();
        __syncwarp();
        if (kPair == 1 && p.ks > 1) {
            // each block of the cluster adds up its share of the tile's columns, a thread some of them of one row
            __syncwarp();
            ptx::cluster_meet();
            const Tile x = tile_of(group);
            const int row = x.i * 128 + lr;
            const long plane = (long)p.S * p.ld_dst;
            for (int c = (rank * 2 + half) * 8, c1 = row < p.S ? 128 : 0; c < c1; c += 16 * p.ks) {
                const int col = x.j * 128 + c;
                if (col >= p.N) break;
                float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (int r = 0; r < p.ks; ++r) {
                    const uint32_t from = ptx::in_block(smem0 + (uint32_t)(c * 128 + lr) * 4, r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float y;
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y) : "r"(from + k * 512) : "memory");
                        v[k] += y;
                    }
                }
                if (kKind == kOrthLast) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] *= p.f;
                    {
                        const size_t step = p.o.tall ? (size_t)p.o.ld_out : 1,
                                     at = x.mat * p.o.step_out + (p.o.tall ? (size_t)col * p.o.ld_out + row : (size_t)row * p.o.ld_out + col);
                        const int n = min(8, p.N - col);
                        if (p.o.w) {
                            float w[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) w[k] = k < n ? to_f32(static_cast<const E *>(p.o.w)[at + k * step]) : 0.f;
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] = fmaf(-p.o.rate, v[k], p.o.keep * w[k]);
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k < n) from_f32(static_cast<E *>(p.o.out)[at + k * step], v[k]);
                    }
                    continue;
                }
                __half *hi = p.dst + 2 * x.mat * plane, *lo = hi + plane;
                if (kKind == kOrthPoly) {
                    const __half *ah = p.a + 2 * x.mat * (long)p.S * p.ld_a + (long)row * p.ld_a + col;
                    float a[8];
                    join8(*reinterpret_cast<const uint4 *>(ah), *reinterpret_cast<const uint4 *>(ah + (long)p.S * p.ld_a), a);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = fmaf(p.fa, a[k], p.f * v[k]) + (row == col + k ? p.fi : 0.f);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] *= p.f;
                }
                uint4 vh, vl;                                            // (ld_dst is a multiple of 8: what is beyond the last column is never read)
                split8(v, vh, vl);
                *reinterpret_cast<uint4 *>(hi + (long)row * p.ld_dst + col) = vh;
                *reinterpret_cast<uint4 *>(lo + (long)row * p.ld_dst + col) = vl;
                if (kSymmetric && x.i != x.j) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (col + k < p.N) split_half(v[k], hi[(long)(col + k) * p.ld_dst + row], lo[(long)(col + k) * p.ld_dst + row]);
                }
            }
            __syncwarp();
        }
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    if (kPair == 2 || p.ks > 1) ptx::cluster_meet();                     // (nobody's shared or tensor memory is needed any more)
    if (threadIdx.x == 0 && abort_flag != 0) p.status[0] = abort_flag;
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_for<kPair>(tmem, 2 * kTileN);
    }
}

// ---------------------------------------------------------------- a whole matrix in one block
// S up to 128 and everything in shared memory: X as panels of 64 columns [ceil(L / 64)][Mr rows][128 bytes] (128-byte swizzle, Mr = S rounded up to
// 16), high halves then low ones, and behind them A, overwritten by B, in the same form.  The same bytes serve as rows of X (sums along
// rows) and as the right factor of B X (sums over rows).  The MMAs have 128 rows whatever S is; rows beyond Mr read what lies behind a
// panel and their sums are not looked at.
struct OrthSmall {
    OrthOuter o;
    OrthScales sc;
    int S, L, Mr, panels, steps;
    uint32_t *status;
};
constexpr int kOrthSmallThreads = 256;
struct OrthSmallSize {
    size_t x_half, a_half, total;
};
__host__ __device__ inline OrthSmallSize orth_small_size(int S, int L) {
    OrthSmallSize z;
    const size_t Mr = (size_t)(S + 15) / 16 * 16;
    z.x_half = (size_t)((L + 63) / 64) * Mr * 128;
    z.a_half = (size_t)((S + 63) / 64) * Mr * 128;
    z.total = 1024 + 2 * (z.x_half + z.a_half) + (128 - Mr) * 128 + 64;     // (what the rows beyond Mr of the last panel read is there)
    return z;
}
// Byte offset of the eight columns from c (a multiple of 8) on of a row.
__device__ __forceinline__ uint32_t panel_at(int row, int c, int Mr) { return (uint32_t)((c >> 6) * Mr + row) * 128 + ((((uint32_t)c >> 3) & 7) ^ (row & 7)) * 16; }

__global__ void __launch_bounds__(kOrthSmallThreads, 1) orth_small_kernel(const OrthSmall p) {
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort_flag;
    __shared__ __align__(8) uint64_t bar_word;
    __shared__ double sums[kOrthSmallThreads / 32];
    uint8_t *smem = ptx::align_1024(raw);
    const OrthSmallSize z = orth_small_size(p.S, p.L);
    uint8_t *xh = smem, *xl = smem + z.x_half, *ah = smem + 2 * z.x_half, *al = ah + z.a_half;
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
    for (size_t i = threadIdx.x; i < (z.total - 1024 - 64) / 16; i += kOrthSmallThreads) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    ptx::grid_launch();
    ptx::grid_wait();
    const OrthOuter &o = p.o;
    double sum = 0.0;
    orth_elements<false>(o, mat, threadIdx.x, kOrthSmallThreads, [&](int, int, const auto &u) {
        for (float x : u) sum += (double)x * x;
    });
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < kOrthSmallThreads / 32; ++k) sum += sums[k];
    const double f = (double)p.sc.x / (sqrt(sum) + (double)o.eps);
    orth_elements<true>(o, mat, threadIdx.x, kOrthSmallThreads, [&](int r, int c, const auto &u) {
        constexpr int V = sizeof(u) / sizeof(float);
        if (V == 4 && !o.tall) {
            uint2 h, l;
            h.x = half_pair((float)(u[0] * f), (float)(u[1 % V] * f), l.x);
            h.y = half_pair((float)(u[2 % V] * f), (float)(u[3 % V] * f), l.y);
            const uint32_t at = panel_at(r, c & ~7, p.Mr) + (c & 7) * 2;
            *reinterpret_cast<uint2 *>(xh + at) = h;
            *reinterpret_cast<uint2 *>(xl + at) = l;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int s = o.tall ? c + i : r, l = o.tall ? r : c + i;
                const uint32_t at = panel_at(s, l & ~7, p.Mr) + (l & 7) * 2;
                split_half((float)(u[i] * f), *reinterpret_cast<__half *>(xh + at), *reinterpret_cast<__half *>(xl + at));
            }
        }
    });
    ptx::fence_proxy_async_smem();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = tmem_slot;

    uint32_t phase = 0;
    constexpr uint32_t hi = ptx::desc_hi(1024, 2);
    const uint32_t dxh = ptx::smem_u32(xh), dxl = ptx::smem_u32(xl), dah = ptx::smem_u32(ah), dal = ptx::smem_u32(al), panel = (uint32_t)p.Mr * 128;
    const int quad = warp & 3, part = warp >> 2, row = quad * 32 + lane, tall_k = p.Mr / 16;
    const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16);
    // the three products of two split factors, one 16-deep step
    auto mma3 = [&](uint32_t d, uint32_t a_hi, uint32_t a_lo, uint32_t b_hi, uint32_t b_lo, uint32_t b_lbo, uint32_t idesc, bool first) {
        ptx::mma_ss(d, ptx::desc(ptx::desc_lo(a_lo, 16), hi), ptx::desc(ptx::desc_lo(b_hi, b_lbo), hi), idesc, !first);
        ptx::mma_ss(d, ptx::desc(ptx::desc_lo(a_hi, 16), hi), ptx::desc(ptx::desc_lo(b_lo, b_lbo), hi), idesc, 1);
        ptx::mma_ss(d, ptx::desc(ptx::desc_lo(a_hi, 16), hi), ptx::desc(ptx::desc_lo(b_hi, b_lbo), hi), idesc, 1);
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
    const int chunk_max = 512;
    bool ok = true;
    for (int step = 0; step < p.steps && ok; ++step) {
        // A = X X^T
        if (warp == 0 && ptx::elect_one()) {
            const uint32_t idesc = instr_desc_f16(128, p.Mr, 0);
            for (int k = 0; k < 4 * p.panels; ++k) {
                const uint32_t at = (k >> 2) * panel + (k & 3) * 32;
                mma3(tmem, dxh + at, dxl + at, dxh + at, dxl + at, 16, idesc, k == 0);
            }
            ptx::mma_commit(bar);
        }
        __syncwarp();
        if (!(ok = finish())) break;
        const float fg = p.sc.a / (p.sc.x * p.sc.x);
        for (int c = part * 16; c < p.Mr; c += 32) {
            uint32_t u[16];
            ptx::tmem_ld16(acc + c, u);
            ptx::tmem_wait_ld();
            if (row < p.Mr) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float v[8];
                    uint4 vh, vl;
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(u[8 * q + k]) * fg;
                    split8(v, vh, vl);
                    const uint32_t at = panel_at(row, c + 8 * q, p.Mr);
                    *reinterpret_cast<uint4 *>(ah + at) = vh;
                    *reinterpret_cast<uint4 *>(al + at) = vl;
                }
            }
        }
        ready();
        // B = a I + b A + c A^2, over A
        if (warp == 0 && ptx::elect_one()) {
            const uint32_t idesc = instr_desc_f16(128, p.Mr, 0);
            for (int k = 0; k < tall_k; ++k) {
                const uint32_t at = (k >> 2) * panel + (k & 3) * 32;
                mma3(tmem, dah + at, dal + at, dah + at, dal + at, 16, idesc, k == 0);
            }
            ptx::mma_commit(bar);
        }
        __syncwarp();
        if (!(ok = finish())) break;
        const float fp = p.sc.cc * p.sc.b / (p.sc.a * p.sc.a), fa = p.sc.cb * p.sc.b / p.sc.a, fi = p.sc.ca * p.sc.b;
        for (int c = part * 16; c < p.Mr; c += 32) {
            uint32_t u[16];
            ptx::tmem_ld16(acc + c, u);
            ptx::tmem_wait_ld();
            if (row < p.Mr) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const uint32_t at = panel_at(row, c + 8 * q, p.Mr);
                    float a[8], v[8];
                    uint4 vh, vl;
                    join8(*reinterpret_cast<const uint4 *>(ah + at), *reinterpret_cast<const uint4 *>(al + at), a);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[k] = fmaf(fa, a[k], fp * __uint_as_float(u[8 * q + k])) + (row == c + 8 * q + k ? fi : 0.f);
                    split8(v, vh, vl);
                    *reinterpret_cast<uint4 *>(ah + at) = vh;
                    *reinterpret_cast<uint4 *>(al + at) = vl;
                }
            }
        }
        ready();
        // X <- B X, as many columns at a time as tensor memory holds
        const float fx = 1.f / p.sc.b;
        for (int l0 = 0; l0 < 64 * p.panels; l0 += chunk_max) {
            const int l1 = min(l0 + chunk_max, 64 * p.panels);
            if (warp == 0 && ptx::elect_one()) {
                for (int l = l0; l < l1; l += 256) {
                    const int w = min(256, l1 - l);
                    const uint32_t idesc = instr_desc_f16(128, w, 1);
                    for (int k = 0; k < tall_k; ++k) {
                        const uint32_t at = (k >> 2) * panel + (k & 3) * 32, bt = (l >> 6) * panel + k * 2048;
                        mma3(tmem + (l - l0), dah + at, dal + at, dxh + bt, dxl + bt, panel, idesc, k == 0);
                    }
                }
                ptx::mma_commit(bar);
            }
            __syncwarp();
            if (!(ok = finish())) break;
            for (int l = l0 + part * 16; l < l1; l += 32) {
                uint32_t u[16];
                ptx::tmem_ld16(acc + (l - l0), u);
                ptx::tmem_wait_ld();
                if (row < p.Mr) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float v[8];
                        uint4 vh, vl;
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(u[8 * q + k]) * fx;
                        split8(v, vh, vl);
                        const uint32_t at = panel_at(row, l + 8 * q, p.Mr);
                        *reinterpret_cast<uint4 *>(xh + at) = vh;
                        *reinterpret_cast<uint4 *>(xl + at) = vl;
                    }
                }
            }
            ready();
        }
    }
    // the result, from its halves
    const float back = 1.f / p.sc.x;
    orth_results(o, mat, threadIdx.x, kOrthSmallThreads, [&](int r, int c, auto &v) {
        constexpr int V = sizeof(v) / sizeof(float);
        auto one = [&](uint32_t at) { return back * (__half2float(*reinterpret_cast<const __half *>(xh + at)) + __half2float(*reinterpret_cast<const __half *>(xl + at))); };
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int s = o.tall ? c + i : r, l = o.tall ? r : c + i;
            v[i] = one(panel_at(s, l & ~7, p.Mr) + (l & 7) * 2);
        }
    });
    ptx::tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag != 0) p.status[0] = abort_flag;
    if (warp == 0) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace flare
