// Norms around a block: the norm before it, and the join after it (norm of the branch, gate, residual scale, sum with the
// residual stream) with the norm before the next block, forward and backward.  Per row (token) of C columns, in float32:
//
//     n  = N_post(o),   y = alpha x + s act(g) n,   h = N_pre(y);      N(v) = (v - mean) rstd w + b,   rstd = 1/sqrt(var + eps)
//
// (rms norms: mean = 0, var = mean square).  Without a branch y = x.  Backward, with u^ the normalised u:
//
//     dt = dy + J_pre^T dh,  dx = alpha dt,  q = act(g) dt,  do = J_post^T (s q),  dg = s act'(g) n dt,
//     J^T d = rstd (d w - mean(d w) - u^ mean(d w u^))                 (rms: without the mean(d w) term)
//     P = sum over rows of q, Q = sum of q o^:   db_post = s P,  dw_post = s Q,  ds = w_post Q + b_post P.
//
// Two sums over rows serve three gradients, and where consecutive rows share a gate row (a group) they are taken of dt
// per group: dg = s act'(g) (w_post Q + b_post P) of the group, and P, Q the sums over groups of act(g) times theirs.
//
// Everything is bound by memory (bfloat16 with a gate: 10 bytes an element forward, 16 backward), so each element is read
// once: a thread owns 8 or 16 columns of a row, a row is held by the next power of two of threads that covers it (up to 512 of a block, wider
// rows by the blocks of a cluster, whose sums meet through distributed shared memory), and the loads of the rows to come are
// in flight in shared memory (cp.async into slots that only the thread itself reads: no barriers).
// Sums over rows stay in the registers of the thread that owns the columns; each block leaves one partial row of them, which a second
// small kernel adds up (in a fixed order).  As many blocks as fit the chip once (256 threads, two a multiprocessor, or 512) take turns of
// neighbouring rows.  Measured, of the copy bandwidth 6549 GB/s: forward 1048576 rows of 128, float32 stream, 287 us (86 %); 16384 rows of
// 4096 with gate and both norms, bfloat16, 120 us (86 %), backward 193 us (85 %); the norm alone, 262144 rows of 128, 26 us (80 %); backward in float32,
// 19946 rows of 200, 30 us (65 %: starts and ends of two kernels, 9 turns).  A quarter of the warps a multiprocessor could hold are there (shared
// memory, registers), so what is left is the chain of a row: wait, sums over threads, barrier.  Deeper rings (4 to 6 stages), streaming stores and
// 32-byte stores changed nothing or up to 3 %.
#pragma once

#include "flare_common.cuh"
#include "flare_ptx.cuh"

namespace flare {

constexpr float kBlockLog2e = 1.4426950408889634f;

struct BlockArgs {
    const void *x, *o, *g, *dy, *dh;                     // x: what the next norm sees (forward: x; backward: y)
    void *y, *h, *dx, *d_o, *dg;
    const float *scale, *w_post, *b_post, *w_pre, *b_pre;
    float4 *stats;                                        // per row: mean and rstd of the branch, mean and rstd of y
    float *part;                                          // partial sums over rows [chunks][sums][C]
    long ld_x, ld_o, ld_g, ld_y, ld_h, ld_dy, ld_dh, ld_dx, ld_do, ld_dg;
    long rows, group;                                     // group: rows that share a gate row (all rows where none is shared)
    int chunks;                                           // blocks per group
    int C, tpr, cluster;                                  // columns, threads of a row in a block (a power of two), blocks of a row
    int has_post, has_pre, layer_post, layer_pre;
    int gate;                                             // 0 none, 1 sigmoid, 2 linear
    int grouped;                                          // gate rows are shared
    float eps_post, eps_pre, alpha, inv_c;
};

// ---------------------------------------------------------------- eight columns
// Pairs of floats: one instruction for two columns.
__device__ __forceinline__ float2 f2(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 f2_fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 f2_mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 f2_add(float2 a, float2 b) { return __fadd2_rn(a, b); }

template <typename E> struct Raw8 { uint4 q[sizeof(E) / 2]; };

__device__ __forceinline__ float2 pair_of(uint32_t v, __nv_bfloat16) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ float2 pair_of(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
__device__ __forceinline__ uint32_t pair_to(float2 v, __nv_bfloat16) { return ptx::pack_bf16(v); }
__device__ __forceinline__ uint32_t pair_to(float2 v, __half) {
    const __half2 h = __float22half2_rn(v);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename E>
__device__ __forceinline__ void unpack8(const Raw8<E> &r, float2 (&f)[4]) {
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[2 * i] = make_float2(__uint_as_float(r.q[i].x), __uint_as_float(r.q[i].y));
            f[2 * i + 1] = make_float2(__uint_as_float(r.q[i].z), __uint_as_float(r.q[i].w));
        }
    } else {
        f[0] = pair_of(r.q[0].x, E{}); f[1] = pair_of(r.q[0].y, E{});
        f[2] = pair_of(r.q[0].z, E{}); f[3] = pair_of(r.q[0].w, E{});
    }
}
template <typename E>
__device__ __forceinline__ Raw8<E> pack8(const float2 (&f)[4]) {
    Raw8<E> r;
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r.q[i] = make_uint4(__float_as_uint(f[2 * i].x), __float_as_uint(f[2 * i].y), __float_as_uint(f[2 * i + 1].x), __float_as_uint(f[2 * i + 1].y));
    } else {
        r.q[0] = make_uint4(pair_to(f[0], E{}), pair_to(f[1], E{}), pair_to(f[2], E{}), pair_to(f[3], E{}));
    }
    return r;
}

// Which eight columns a thread owns, and how they are moved.  kEight: next to each other, 16 bytes at a time (C a multiple of 8, rows on 16-byte
// boundaries, 16-bit types).  kFours: the same with a float32 stream: two fours, the second behind the first fours of all of the row's threads, so that
// 16 bytes of neighbouring lanes are next to each other in float32 and 8 in a 16-bit type.  kEach: every 32nd of the warp's 256, one at a time
// (a distance the compiler knows: it goes into the instructions).
// (Eight in a row of float32, lanes 32 bytes apart, touch every sector twice: 1048576 rows of 128 forward 340 us instead of 289, 19946 rows of 200
// with gate and post norm backward 41.2 instead of 29.8.)
enum { kEach = 0, kEight = 1, kFours = 2 };
template <typename R, bool kAligned> __host__ __device__ constexpr int move_of() { return !kAligned ? kEach : sizeof(R) == 4 ? kFours : kEight; }
template <int kMove>
struct Columns {
    int first, apart, C;                                     // apart: from the first four to the second
    int mine;                                                // how many of the eight there are (kFours: none or the first four at least)
    __device__ __forceinline__ Columns() {}
    // of the lane-th thread of a row; base: columns before its first
    __device__ __forceinline__ Columns(int lane, int tpr, int C_, int base) : apart(kMove == kFours ? 4 * tpr : 4), C(C_) {
        first = base + (kMove == kEight ? 8 * lane : kMove == kFours ? 4 * lane : 8 * (lane & ~31) + (lane & 31));
        mine = kMove == kEach ? max(0, min(8, (C - first + 31) >> 5)) : first < C ? 8 : 0;
    }
    __device__ __forceinline__ int at(int j) const { return first + (kMove == kEach ? j * 32 : kMove == kEight ? j : (j & 3) + (j >> 2) * apart); }
    __device__ __forceinline__ bool four(int i) const { return kMove == kFours && i == 1 ? first + apart < C : mine > 0; }
    __device__ __forceinline__ bool has(int j) const { return kMove == kFours ? four(j >> 2) : j < mine; }
    // where a row's copy begins: the thread's first column (0 where it has none), of kEach its warp's (the base is a multiple of 256)
    __device__ __forceinline__ int from() const { return kMove == kEach ? first & ~255 : mine > 0 ? first : 0; }
};
template <typename E, int kMove>
__device__ __forceinline__ Raw8<E> load8(const E *row, const Columns<kMove> &c) {
    Raw8<E> r;
    if constexpr (kMove == kEach) {
        float2 f[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) (&f[j / 2].x)[j & 1] = c.has(j) ? to_f32(row[c.at(j)]) : 0.f;
        r = pack8<E>(f);
    } else if constexpr (kMove == kFours && sizeof(E) == 2) {
        const uint2 lo = c.four(0) ? *reinterpret_cast<const uint2 *>(row + c.at(0)) : make_uint2(0, 0), hi = c.four(1) ? *reinterpret_cast<const uint2 *>(row + c.at(4)) : make_uint2(0, 0);
        r.q[0] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(E) / 2; ++i) r.q[i] = c.four(i) ? *reinterpret_cast<const uint4 *>(row + c.at(4 * i)) : make_uint4(0, 0, 0, 0);
    }
    return r;
}
template <typename E, int kMove>
__device__ __forceinline__ void store8(E *row, const Columns<kMove> &c, const float2 (&f)[4]) {
    if constexpr (kMove == kEach) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.has(j)) from_f32(row[c.at(j)], (&f[j / 2].x)[j & 1]);
    } else {
        const Raw8<E> r = pack8<E>(f);
        if constexpr (kMove == kFours && sizeof(E) == 2) {
            if (c.four(0)) *reinterpret_cast<uint2 *>(row + c.at(0)) = make_uint2(r.q[0].x, r.q[0].y);
            if (c.four(1)) *reinterpret_cast<uint2 *>(row + c.at(4)) = make_uint2(r.q[0].z, r.q[0].w);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(E) / 2; ++i)
                if (c.four(i)) *reinterpret_cast<uint4 *>(row + c.at(4 * i)) = r.q[i];
        }
    }
}
// A parameter's eight values; `none` where it is absent, 0 beyond the last column.
template <int kMove>
__device__ __forceinline__ void load_param(const float *p, float none, const Columns<kMove> &c, float2 (&f)[4]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) (&f[j / 2].x)[j & 1] = !c.has(j) ? 0.f : p ? p[c.at(j)] : none;
}

// ---------------------------------------------------------------- sums over the threads of a row
struct RowShared {
    float4 warp[2][16];         // what the warps of a row leave for one another, two buffers in turn: one barrier a sum
    float4 block[2][8];         // what the blocks of a cluster do
};
struct RowShared8 {
    float warp[2][16][8], block[2][8][8];                    // the same of several sums at once
};
struct RowGroup {
    int tpr, warps, first;      // threads and warps of a row in the block, the row's first warp
    int warp;                   // this thread's warp
    int cluster;                // blocks of a row
    int turn;
    RowShared *sh;
    RowShared8 *sh8;
    __device__ __forceinline__ RowGroup(int tpr_, int cluster_, RowShared *sh_, RowShared8 *sh8_ = nullptr) : tpr(tpr_), cluster(cluster_), turn(0), sh(sh_), sh8(sh8_) {
        warp = threadIdx.x >> 5;
        warps = tpr > 32 ? tpr >> 5 : 1;
        first = warp & ~(warps - 1);
        if (cluster > 1) meet();                             // (the other blocks' shared memory is there from here on)
    }
    __device__ __forceinline__ void meet() const {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    // Sum over the lanes whose indexes differ below n (a power of two), in each of them.
    __device__ __forceinline__ static float over(float v, int n) {
        if (n == 32) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        } else {
#pragma unroll
            for (int o = 8; o > 0; o >>= 1)
                if (n > o) v += __shfl_xor_sync(0xffffffffu, v, o);
        }
        return v;
    }
    __device__ __forceinline__ float within_warp(float v) const { return over(v, min(tpr, 32)); }
    // v of every warp of the row in this block: in lane k that of the (k mod warps)-th.  All threads of the block call it: a barrier of the row's own
    // threads, so that rows need not wait for one another, measured slower (backward of 4096 columns 122 us instead of 113).
    __device__ __forceinline__ float4 of_warps(float4 v) {
        if ((threadIdx.x & 31) == 0) sh->warp[turn][warp] = v;
        __syncthreads();
        return sh->warp[turn][first + (threadIdx.x & (warps - 1))];
    }
    // v (the same in all threads of a block) of every block of the row: in lane k that of the (k mod cluster)-th.  All threads of the cluster call it.
    __device__ __forceinline__ float4 of_blocks(float4 v) {
        if ((int)threadIdx.x < cluster) {
            uint32_t to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(ptx::smem_u32(&sh->block[turn][blockIdx.y])), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
        }
        meet();
        return sh->block[turn][threadIdx.x & (cluster - 1)];
    }
    // Sums of a and, if kTwo, b over the row.  All threads of the block (and its cluster) call it.
    template <bool kTwo>
    __device__ __forceinline__ float2 sum(float a, float b) {
        a = within_warp(a);
        if (kTwo) b = within_warp(b);
        if (tpr > 32) {
            float4 v = of_warps(make_float4(a, b, 0.f, 0.f));
            a = over(v.x, warps);
            if (kTwo) b = over(v.y, warps);
            if (cluster > 1) {
                v = of_blocks(make_float4(a, b, 0.f, 0.f));
                a = over(v.x, cluster);
                if (kTwo) b = over(v.y, cluster);
            }
            turn ^= 1;
        }
        return make_float2(a, b);
    }
    // Sums of kN values (4 or 8) over a row of more than one warp, in one round.  In a warp every step halves the values a lane has, so that kN + 1 or kN
    // + 2 shuffles do what kN times five would.  All threads of the block (and its cluster) call it.
    template <int kN>
    __device__ __forceinline__ void sums(float (&v)[kN]) {
        const int l = threadIdx.x & 31, of = l % kN;
        int at = 0;                                          // which of the values this lane is left with
#pragma unroll
        for (int n = kN / 2, o = 16; n > 0; n /= 2, o /= 2) {
            const bool upper = l & o;
            at = 2 * at + (upper ? 1 : 0);
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float keep = upper ? v[i + n] : v[i], give = upper ? v[i] : v[i + n];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        }
        float mine = over(v[0], 32 / kN);
        if ((l & (32 / kN - 1)) == 0) sh8->warp[turn][warp][at] = mine;
        __syncthreads();
        mine = 0.f;
        for (int k = l / kN; k < warps; k += 32 / kN) mine += sh8->warp[turn][first + k][of];
#pragma unroll
        for (int o = kN; o < 32; o *= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        if (cluster > 1) {
            if (warp == 0)
                for (int k = l / kN; k < cluster; k += 32 / kN) {
                    uint32_t to;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(ptx::smem_u32(&sh8->block[turn][blockIdx.y][of])), "r"(k));
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(mine) : "memory");
                }
            meet();
            mine = 0.f;
            for (int k = l / kN; k < cluster; k += 32 / kN) mine += sh8->block[turn][k][of];
#pragma unroll
            for (int o = kN; o < 32; o *= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        }
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = __shfl_sync(0xffffffffu, mine, i);
    }
    // (sum, squares of distances from the own mean, own mean, count) in n lanes -> the same of their union, of 1 / inv elements
    __device__ __forceinline__ static float4 join_parts(float4 v, int n, float inv, float count) {
        const float sum = over(v.x, n), mean = sum * inv, d = v.z - mean;
        return make_float4(sum, over(fmaf(v.w * d, d, v.y), n), mean, count);
    }
};

// How many elements of a row a warp and a block have.
struct RowCounts {
    float warp, block, inv_warp, inv_block;                  // (the inverse of none: 0)
    __device__ __forceinline__ RowCounts(RowGroup &grp, int C, int mine, int block_first, int block_columns) {
        warp = grp.within_warp((float)mine);
        block = (float)max(0, min(C - block_first, block_columns));
        inv_warp = warp > 0.f ? 1.f / warp : 0.f;
        inv_block = block > 0.f ? 1.f / block : 0.f;
    }
};

// Mean and 1/sqrt(var + eps) of a row.  layer: the squares are of distances from the mean, first the warp's, put together with those of the
// row's other warps by the distances of their means (one barrier, and no small difference of large sums).
template <int kV, int kMove>
__device__ __forceinline__ float2 moments(RowGroup &grp, const float2 (&v)[kV][4], const Columns<kMove> *c, const RowCounts &n, int layer, float inv_c, float eps) {
    if (!layer) {
        float2 s = f2(0.f);
#pragma unroll
        for (int g = 0; g < kV; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) s = f2_fma(v[g][i], v[g][i], s);
        const float sq = grp.sum<false>(s.x + s.y, 0.f).x;
        return make_float2(0.f, rsqrtf(fmaf(sq, inv_c, eps)));
    }
    float2 t = f2(0.f);
#pragma unroll
    for (int g = 0; g < kV; ++g) t = f2_add(t, f2_add(f2_add(v[g][0], v[g][1]), f2_add(v[g][2], v[g][3])));
    const float sum = grp.within_warp(t.x + t.y);
    const float mean_w = sum * n.inv_warp;
    float m2 = 0.f;
#pragma unroll
    for (int g = 0; g < kV; ++g) {
        if constexpr (kMove == kEach) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = c[g].has(j) ? (&v[g][j / 2].x)[j & 1] - mean_w : 0.f;
                m2 = fmaf(d, d, m2);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float2 d0 = f2_add(v[g][2 * q], f2(-mean_w)), d1 = f2_add(v[g][2 * q + 1], f2(-mean_w)), s = f2_fma(d1, d1, f2_mul(d0, d0));
                m2 += c[g].four(q) ? s.x + s.y : 0.f;
            }
        }
    }
    m2 = grp.within_warp(m2);
    float4 part = make_float4(sum, m2, mean_w, n.warp);
    if (grp.tpr > 32) {
        part = RowGroup::join_parts(grp.of_warps(part), grp.warps, n.inv_block, n.block);
        if (grp.cluster > 1) part = RowGroup::join_parts(grp.of_blocks(part), grp.cluster, inv_c, 0.f);
        grp.turn ^= 1;
    }
    return make_float2(part.z, rsqrtf(fmaf(part.y, inv_c, eps)));
}

// (The exponent is a product that is rounded once, and so is log2 e: a is off by some 1e-7 |g| of itself, also for float32 gates.)
__device__ __forceinline__ float gate_act(int kind, float g) {
    if (kind != 1) return g;
    float a;                                                 // (of 1 + exp(-g) = infinity: 0)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(1.f + ptx::ex2(-kBlockLog2e * g)));
    return a;
}

__device__ __forceinline__ void gate_act8(int kind, float2 (&a)[4]) {
    if (kind == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = make_float2(gate_act(1, a[i].x), gate_act(1, a[i].y));
    }
}

// ---------------------------------------------------------------- loads ahead
// Slots of kStages rows ahead in shared memory, [stage][16-byte piece][thread]: a thread copies into its own and reads only those.
__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src, bool yes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(yes ? 16u : 0u) : "memory");
}
template <typename E, int kThreads, int kMove>
__device__ __forceinline__ void slot_copy(uint32_t slot, const char *src, const Columns<kMove> &c, bool yes) {      // src: of the first column; yes: and it is one of ours
    if constexpr (kMove == kFours && sizeof(E) == 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(slot + 8 * i), "l"(src + i * c.apart * 2), "r"(yes && (i == 0 || c.four(i)) ? 8u : 0u) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(E) / 2; ++i) copy_async16(slot + i * kThreads * 16, src + i * c.apart * (int)sizeof(E), yes && (i == 0 || c.four(i)));
    }
}
template <typename E, int kThreads>
__device__ __forceinline__ Raw8<E> slot_read(uint32_t slot) {
    Raw8<E> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(E) / 2; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.q[i].x), "=r"(r.q[i].y), "=r"(r.q[i].z), "=r"(r.q[i].w) : "r"(slot + i * kThreads * 16) : "memory");
    return r;
}

// Rows off 16-byte boundaries (40028 rows of 333, float16 with a float32 stream, backward: 45 us; 58 with a word asked for per column): a warp copies the aligned 16-byte pieces that its 256 columns lie in, one more than they fill, and its lanes read their
// columns from there (neighbouring lanes neighbouring columns).  What of the first piece is before the row is not used: it shares an aligned 16 bytes with
// an element of the tensor, so it is in the same allocation.  What is behind the row's end is not read but filled with zeros.
__device__ __forceinline__ uint32_t shift_of(const void *t, long row, long ld, int size) {      // bytes of its first piece that are before the row
    return ((uint32_t)reinterpret_cast<uintptr_t>(t) + (uint32_t)row * (uint32_t)ld * (uint32_t)size) & 15u;
}
template <typename E>
__device__ __forceinline__ void warp_copy(uint32_t slot, const char *src, int bytes) {          // bytes: of the row from src on, 0 or less for none
    constexpr int kBytes = 256 * (int)sizeof(E);
    const int lane = threadIdx.x & 31;
    const uint32_t shift = (uint32_t)reinterpret_cast<uintptr_t>(src) & 15u;
    const int left = bytes > 0 ? min(bytes, kBytes) + (int)shift - 16 * lane : 0;
    src += 16 * lane - (int)shift;
    slot += 16 * lane;
#pragma unroll
    for (int i = 0; i <= kBytes / 512; ++i)
        if (i < kBytes / 512 || lane == 0)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot + 512 * i), "l"(src + 512 * i), "r"(max(0, min(16, left - 512 * i))) : "memory");
}
template <typename E>
__device__ __forceinline__ void warp_read(uint32_t slot, uint32_t shift, float2 (&f)[4]) {
    slot += shift + (threadIdx.x & 31) * (uint32_t)sizeof(E);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float x;
        if constexpr (sizeof(E) == 4) {
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(slot + j * 128) : "memory");
        } else {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(slot + j * 64) : "memory");
            x = pair_of(v, E{}).x;
        }
        (&f[j / 2].x)[j & 1] = x;
    }
}

template <int kThreads>
__device__ __forceinline__ void slot_write(uint32_t slot, const float2 (&f)[4]) {
    const Raw8<float> r = pack8<float>(f);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(slot + i * kThreads * 16), "r"(r.q[i].x), "r"(r.q[i].y), "r"(r.q[i].z), "r"(r.q[i].w) : "memory");
}

// What comes in beside the residual stream: nothing, a branch, a branch with a gate row a row, a branch with gate rows that are shared.
enum { kAlone = 0, kPlain = 1, kGated = 2, kShared = 3 };
// 16-byte pieces of eight columns of everything that is loaded.
template <typename E> __host__ __device__ constexpr int pieces_of() { return (int)sizeof(E) / 2; }
template <typename T, typename R, int kIn> __host__ __device__ constexpr int fwd_pieces() {
    return pieces_of<R>() + (kIn == kAlone ? 0 : kIn == kGated ? 2 : 1) * pieces_of<T>();
}
template <typename T, typename R, int kIn> __host__ __device__ constexpr int bwd_pieces() {
    return 2 * pieces_of<R>() + (kIn == kAlone ? 1 : kIn == kGated ? 3 : 2) * pieces_of<T>();
}
// Bytes of a block's slots of one tensor (off 16-byte boundaries: a piece more a warp), and of all of them for one turn.
template <typename E, bool kAligned, int kThreads> __host__ __device__ constexpr int slots_of() { return pieces_of<E>() * kThreads * 16 + (kAligned ? 0 : kThreads / 2); }
template <typename T, typename R, bool kAligned, int kIn, int kV, int kThreads> __host__ __device__ constexpr int fwd_stage() {
    return kV * (slots_of<R, kAligned, kThreads>() + (kIn == kAlone ? 0 : kIn == kGated ? 2 : 1) * slots_of<T, kAligned, kThreads>());
}
template <typename T, typename R, bool kAligned, int kIn, int kV, int kThreads> __host__ __device__ constexpr int bwd_stage() {
    return kV * (2 * slots_of<R, kAligned, kThreads>() + (kIn == kAlone ? 1 : kIn == kGated ? 3 : 2) * slots_of<T, kAligned, kThreads>());
}
__host__ __device__ constexpr int stages_for(int pieces) { return pieces <= 3 ? 4 : pieces <= 7 ? 3 : 2; }

// The rows of one block: every chunks-th turn of `turn` rows of a group (so that the blocks at work at a time are at neighbouring rows).
struct Piece {
    long begin, end, group;
    int step;
    __device__ __forceinline__ Piece(const BlockArgs &p, int turn) {
        group = blockIdx.x / p.chunks;
        begin = group * p.group + (blockIdx.x - group * p.chunks) * turn;
        end = (group + 1) * p.group;
        step = turn * p.chunks;
    }
};

// ---------------------------------------------------------------- forward
// kV: groups of eight columns a thread owns.  With two, what a row costs beside its elements (sums over its threads, addresses) counts half; the
// biases are then kept in shared memory, where only their own thread reads them.
template <typename T, typename R, bool kAligned, int kIn, bool kBias, int kV, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : 2) block_forward_kernel(BlockArgs p) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ RowShared row_shared;
    constexpr bool kBranch = kIn != kAlone;
    constexpr int kStages = stages_for(fwd_pieces<T, R, kIn>() * kV);
    constexpr uint32_t kSlotR = slots_of<R, kAligned, kThreads>(), kSlotT = slots_of<T, kAligned, kThreads>();
    constexpr uint32_t kX = 0, kO = kV * kSlotR, kG = kO + kV * kSlotT, kStage = fwd_stage<T, R, kAligned, kIn, kV, kThreads>();
    const int lane = threadIdx.x & (p.tpr - 1), per_turn = kThreads / p.tpr, mine = threadIdx.x / p.tpr;
    constexpr int kMove = move_of<R, kAligned>();
    Columns<kMove> c[kV];
    int mine_n = 0;
#pragma unroll
    for (int g = 0; g < kV; ++g) {
        c[g] = Columns<kMove>(lane, p.tpr, p.C, blockIdx.y * 8 * kV * kThreads + g * 8 * p.tpr);
#pragma unroll
        for (int j = 0; j < 8; ++j) mine_n += c[g].has(j) ? 1 : 0;
    }
    RowGroup grp(p.tpr, p.cluster, &row_shared);
    const Piece piece(p, per_turn);
    constexpr bool gate_row = kIn == kGated;
    const RowCounts counts(grp, p.C, mine_n, blockIdx.y * 8 * kV * kThreads, 8 * kV * kThreads);
    ptx::grid_launch();
    ptx::grid_wait();

    constexpr bool kBiasSlots = kBias && kV == 2;
    const uint32_t slots = ptx::smem_u32(smem) + (kAligned ? threadIdx.x * 16 : 0), bias_slots = slots + kStages * kStage;   // [post, pre][group][half][thread]
    float2 sw[kV][4], sb[kV][4], w[kV][4], b[kV][4], a[kV][4];
#pragma unroll
    for (int g = 0; g < kV; ++g) {
        if constexpr (kBranch) {
            float2 s[4];
            load_param(p.scale, 1.f, c[g], s);
            load_param(p.w_post, 1.f, c[g], sw[g]);
            if constexpr (kBias) load_param(p.b_post, 0.f, c[g], sb[g]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sw[g][i] = f2_mul(sw[g][i], s[i]);
                if constexpr (kBias) sb[g][i] = f2_mul(sb[g][i], s[i]);
                a[g][i] = f2(1.f);
            }
            if constexpr (kIn == kShared) {
                unpack8(load8(static_cast<const T *>(p.g) + piece.group * p.ld_g, c[g]), a[g]);
                gate_act8(p.gate, a[g]);
            }
        }
        load_param(p.w_pre, 1.f, c[g], w[g]);
        if constexpr (kBias) load_param(p.b_pre, 0.f, c[g], b[g]);
        if constexpr (kBiasSlots) {
            if constexpr (kBranch) slot_write<kThreads>(bias_slots + g * 2 * kThreads * 16, sb[g]);
            slot_write<kThreads>(bias_slots + (kV + g) * 2 * kThreads * 16, b[g]);
        }
    }

    // loads run kStages - 1 turns ahead of the rows: pointers to the next row to ask for, and rows left from there
    const char *from_x = nullptr, *from_o = nullptr, *from_g = nullptr;
    const long row0 = piece.begin + mine, step_x = piece.step * p.ld_x * (long)sizeof(R), step_o = piece.step * p.ld_o * (long)sizeof(T), step_g = piece.step * p.ld_g * (long)sizeof(T);
    const int columns = c[0].from(), apart = 8 * p.tpr;
    const uint32_t warp_r = (threadIdx.x >> 5) * (kSlotR / (kThreads / 32)), warp_t = (threadIdx.x >> 5) * (kSlotT / (kThreads / 32));   // (off boundaries: a warp's slots)
    int ahead = (int)(piece.end - row0);
    from_x = reinterpret_cast<const char *>(static_cast<const R *>(p.x) + row0 * p.ld_x + columns);
    if constexpr (kBranch) {
        from_o = reinterpret_cast<const char *>(static_cast<const T *>(p.o) + row0 * p.ld_o + columns);
        if constexpr (gate_row) from_g = reinterpret_cast<const char *>(static_cast<const T *>(p.g) + row0 * p.ld_g + columns);
    }
    auto fetch = [&](int stage) {
        if constexpr (kAligned) {
            const uint32_t s = slots + stage * kStage;
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                const bool yes = ahead > 0 && c[g].four(0);
                slot_copy<R, kThreads>(s + kX + g * kSlotR, from_x + g * apart * (int)sizeof(R), c[g], yes);
                if constexpr (kBranch) {
                    slot_copy<T, kThreads>(s + kO + g * kSlotT, from_o + g * apart * (int)sizeof(T), c[g], yes);
                    if constexpr (gate_row) slot_copy<T, kThreads>(s + kG + g * kSlotT, from_g + g * apart * (int)sizeof(T), c[g], yes);
                }
            }
        } else {
            const uint32_t s = slots + stage * kStage;
            const int left = ahead > 0 ? p.C - columns : 0;
            warp_copy<R>(s + kX + warp_r, from_x, left * (int)sizeof(R));
            if constexpr (kBranch) warp_copy<T>(s + kO + warp_t, from_o, left * (int)sizeof(T));
            if constexpr (gate_row) warp_copy<T>(s + kG + warp_t, from_g, left * (int)sizeof(T));
        }
        ptx::copy_async_commit();
        ahead -= piece.step;
        from_x += step_x;
        if constexpr (kBranch) from_o += step_o;
        if constexpr (gate_row) from_g += step_g;
    };
    for (int k = 0; k < kStages - 1; ++k) fetch(k);

    int stage = 0;
    for (long row = row0; row - mine < piece.end; row += piece.step) {
        const bool live = row < piece.end;
        float2 y[kV][4];
        const uint32_t s = slots + stage * kStage;
        if constexpr (!kAligned) __syncwarp();               // (the other lanes have read the slots that are filled now)
        fetch(stage == 0 ? kStages - 1 : stage - 1);
        ptx::copy_async_wait<kStages - 1>();
        if constexpr (!kAligned) __syncwarp();               // (and what they copied is there)
#pragma unroll
        for (int g = 0; g < kV; ++g) {
            if constexpr (kAligned) unpack8(slot_read<R, kThreads>(s + kX + g * kSlotR), y[g]);
            else warp_read<R>(s + kX + warp_r, shift_of(p.x, row, p.ld_x, sizeof(R)), y[g]);
        }
        float2 st_o = make_float2(0.f, 0.f);
        if constexpr (kBranch) {
            float2 o[kV][4];
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                if constexpr (kAligned) {
                    unpack8(slot_read<T, kThreads>(s + kO + g * kSlotT), o[g]);
                    if constexpr (gate_row) unpack8(slot_read<T, kThreads>(s + kG + g * kSlotT), a[g]);
                } else {
                    warp_read<T>(s + kO + warp_t, shift_of(p.o, row, p.ld_o, sizeof(T)), o[g]);
                    if constexpr (gate_row) warp_read<T>(s + kG + warp_t, shift_of(p.g, row, p.ld_g, sizeof(T)), a[g]);
                }
                if constexpr (gate_row) gate_act8(p.gate, a[g]);
            }
            if (p.has_post) st_o = moments<kV>(grp, o, c, counts, p.layer_post, p.inv_c, p.eps_post);
            const float mean = -st_o.x, rstd = p.has_post ? st_o.y : 1.f;
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                if constexpr (kBiasSlots) unpack8(slot_read<float, kThreads>(bias_slots + g * 2 * kThreads * 16), sb[g]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 n = f2_mul(f2_add(o[g][i], f2(mean)), f2(rstd));
                    const float2 v = kBias ? f2_fma(n, sw[g][i], sb[g][i]) : f2_mul(n, sw[g][i]);
                    y[g][i] = f2_fma(y[g][i], f2(p.alpha), kIn == kPlain ? v : f2_mul(v, a[g][i]));
                }
                if (live) store8(static_cast<R *>(p.y) + row * p.ld_y, c[g], y[g]);
            }
        }
        float2 st_y = make_float2(0.f, 0.f);
        if (p.has_pre) {
            st_y = moments<kV>(grp, y, c, counts, p.layer_pre, p.inv_c, p.eps_pre);
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                if constexpr (kBiasSlots) unpack8(slot_read<float, kThreads>(bias_slots + (kV + g) * 2 * kThreads * 16), b[g]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 n = f2_mul(f2_add(y[g][i], f2(-st_y.x)), f2(st_y.y));
                    y[g][i] = kBias ? f2_fma(n, w[g][i], b[g][i]) : f2_mul(n, w[g][i]);
                }
                if (live) store8(static_cast<T *>(p.h) + row * p.ld_h, c[g], y[g]);
            }
        }
        if (live && lane == 0 && blockIdx.y == 0 && p.stats) p.stats[row] = make_float4(st_o.x, st_o.y, st_y.x, st_y.y);
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
}

// ---------------------------------------------------------------- backward
// Sums over rows: [0] dh y^, [1] Q, [2] dh, [3] P; without biases the first two, without a branch [0] and [2].
template <bool kBranch, bool kBias> __host__ __device__ constexpr int bwd_sums() { return (kBranch ? 2 : 1) * (kBias ? 2 : 1); }

template <typename T, typename R, bool kAligned, int kIn, bool kBias, bool kOnce, int kV, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : 2) block_backward_kernel(BlockArgs p) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ RowShared row_shared;
    constexpr bool kBranch = kIn != kAlone;
    constexpr int kStages = stages_for(bwd_pieces<T, R, kIn>() * kV), kSums = bwd_sums<kBranch, kBias>();
    constexpr uint32_t kOneR = slots_of<R, kAligned, kThreads>(), kOneT = slots_of<T, kAligned, kThreads>();
    constexpr uint32_t kY = 0, kDy = kV * kOneR, kDh = 2 * kDy, kO = kDh + kV * kOneT, kG = kO + kV * kOneT, kStage = bwd_stage<T, R, kAligned, kIn, kV, kThreads>();
    const int lane = threadIdx.x & (p.tpr - 1), per_turn = kThreads / p.tpr, mine = threadIdx.x / p.tpr;
    constexpr int kMove = move_of<R, kAligned>();
    Columns<kMove> c[kV];
#pragma unroll
    for (int g = 0; g < kV; ++g) c[g] = Columns<kMove>(lane, p.tpr, p.C, blockIdx.y * 8 * kV * kThreads + g * 8 * p.tpr);
    RowShared8 *row_shared8 = nullptr;
    if constexpr (kOnce) {                                   // (two blocks of the widest form fit an SM to the last KB)
        __shared__ RowShared8 eight;
        row_shared8 = &eight;
    }
    RowGroup grp(p.tpr, p.cluster, &row_shared, row_shared8);
    const Piece piece(p, per_turn);
    constexpr bool gate_row = kIn == kGated;
    ptx::grid_launch();
    ptx::grid_wait();

    // two groups of columns: the weights in shared memory (w, sw) leave the registers for the sums
    constexpr bool kWeightSlots = kV == 2 && (kBranch || kBias);
    constexpr uint32_t kWeights = kV * 2 * kThreads * 16;
    const uint32_t slots = ptx::smem_u32(smem) + (kAligned ? threadIdx.x * 16 : 0), weight_slots = slots + kStages * kStage;
    float2 sw[kV][4], sb[kV][4], w[kV][4], a[kV][4], sum[kSums][kV][4];
#pragma unroll
    for (int g = 0; g < kV; ++g) {
        if constexpr (kBranch) {
            float2 s[4];
            load_param(p.scale, 1.f, c[g], s);
            load_param(p.w_post, 1.f, c[g], sw[g]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sw[g][i] = f2_mul(sw[g][i], s[i]);
                a[g][i] = f2(1.f);
            }
            if constexpr (kBias) {
                load_param(p.b_post, 0.f, c[g], sb[g]);
#pragma unroll
                for (int i = 0; i < 4; ++i) sb[g][i] = f2_mul(sb[g][i], s[i]);
            }
            if constexpr (kIn == kShared) {
                unpack8(load8(static_cast<const T *>(p.g) + piece.group * p.ld_g, c[g]), a[g]);
                gate_act8(p.gate, a[g]);
            }
        }
        load_param(p.w_pre, 1.f, c[g], w[g]);
        if constexpr (kWeightSlots) {
            slot_write<kThreads>(weight_slots + g * 2 * kThreads * 16, w[g]);
            if constexpr (kBranch) slot_write<kThreads>(weight_slots + kWeights + g * 2 * kThreads * 16, sw[g]);
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[k][g][i] = f2(0.f);
    }

    // loads run kStages - 1 turns ahead of the rows: pointers to the next row to ask for, and rows left from there
    const uint32_t warp_r = (threadIdx.x >> 5) * (kOneR / (kThreads / 32)), warp_t = (threadIdx.x >> 5) * (kOneT / (kThreads / 32));     // (off boundaries: a warp's slots)
    const char *from_y = nullptr, *from_dy = nullptr, *from_dh = nullptr, *from_o = nullptr, *from_g = nullptr;
    const long first = piece.begin + mine;
    int ahead = (int)(piece.end - first);
    const int columns = c[0].from(), apart = 8 * p.tpr;
    {
        auto at = [&](const void *t, long ld, size_t size) { return static_cast<const char *>(t) + (first * ld + columns) * (long)size; };
        from_y = at(p.x, p.ld_x, sizeof(R)); from_dy = at(p.dy, p.ld_dy, sizeof(R)); from_dh = at(p.dh, p.ld_dh, sizeof(T));
        if constexpr (kBranch) from_o = at(p.o, p.ld_o, sizeof(T));
        if constexpr (gate_row) from_g = at(p.g, p.ld_g, sizeof(T));
    }
    auto fetch = [&](int stage) {
        if constexpr (kAligned) {
            const uint32_t s = slots + stage * kStage;
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                const bool yes = ahead > 0 && c[g].four(0);
                if (p.has_pre) {
                    slot_copy<R, kThreads>(s + kY + g * kOneR, from_y + g * apart * (int)sizeof(R), c[g], yes);
                    slot_copy<T, kThreads>(s + kDh + g * kOneT, from_dh + g * apart * (int)sizeof(T), c[g], yes);
                }
                if (p.dy) slot_copy<R, kThreads>(s + kDy + g * kOneR, from_dy + g * apart * (int)sizeof(R), c[g], yes);
                if constexpr (kBranch) {
                    slot_copy<T, kThreads>(s + kO + g * kOneT, from_o + g * apart * (int)sizeof(T), c[g], yes);
                    if constexpr (gate_row) slot_copy<T, kThreads>(s + kG + g * kOneT, from_g + g * apart * (int)sizeof(T), c[g], yes);
                }
            }
        } else {
            const uint32_t s = slots + stage * kStage;
            const int left = ahead > 0 ? p.C - columns : 0;
            if (p.has_pre) {
                warp_copy<R>(s + kY + warp_r, from_y, left * (int)sizeof(R));
                warp_copy<T>(s + kDh + warp_t, from_dh, left * (int)sizeof(T));
            }
            if (p.dy) warp_copy<R>(s + kDy + warp_r, from_dy, left * (int)sizeof(R));
            if constexpr (kBranch) warp_copy<T>(s + kO + warp_t, from_o, left * (int)sizeof(T));
            if constexpr (gate_row) warp_copy<T>(s + kG + warp_t, from_g, left * (int)sizeof(T));
        }
        ptx::copy_async_commit();
        ahead -= piece.step;
        from_y += piece.step * p.ld_x * (long)sizeof(R); from_dy += piece.step * p.ld_dy * (long)sizeof(R); from_dh += piece.step * p.ld_dh * (long)sizeof(T);
        if constexpr (kBranch) from_o += piece.step * p.ld_o * (long)sizeof(T);
        if constexpr (gate_row) from_g += piece.step * p.ld_g * (long)sizeof(T);
    };
    for (int k = 0; k < kStages - 1; ++k) fetch(k);
    const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
    float4 st_next = piece.begin + mine < piece.end ? p.stats[piece.begin + mine] : none;

    int stage = 0;
    for (long r0 = piece.begin; r0 < piece.end; r0 += piece.step) {
        const long row = r0 + mine;
        const bool live = row < piece.end;
        const float4 st = st_next;
        if (row + piece.step < piece.end) st_next = p.stats[row + piece.step];
        else st_next = none;
        const uint32_t s0 = slots + stage * kStage;
        if constexpr (!kAligned) __syncwarp();               // (as in the forward)
        fetch(stage == 0 ? kStages - 1 : stage - 1);
        ptx::copy_async_wait<kStages - 1>();
        if constexpr (!kAligned) __syncwarp();
        auto read = [&](auto type, uint32_t slot, uint32_t warp_slot, int g, const void *t, long ld, float2 (&f)[4]) {
            using E = decltype(type);
            if constexpr (kAligned) unpack8(slot_read<E, kThreads>(s0 + slot + g * slots_of<E, kAligned, kThreads>()), f);
            else warp_read<E>(s0 + slot + warp_slot, shift_of(t, row, ld, sizeof(E)), f);
        };
        float2 dt[kV][4];
#pragma unroll
        for (int g = 0; g < kV; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) dt[g][i] = f2(0.f);
            if (p.dy) read(R{}, kDy, warp_r, g, p.dy, p.ld_dy, dt[g]);
        }
        [[maybe_unused]] float2 o[kV][4], post_means = make_float2(0.f, 0.f);
        if constexpr (kOnce) {
            // (d1 and d2 below are linear in the means that dt is made with: all sums in one round)
            float2 yh[kV][4], c1 = f2(0.f), c2 = f2(0.f), za = f2(0.f), zy = f2(0.f), z1 = f2(0.f), sa = f2(0.f), sy = f2(0.f), s1 = f2(0.f);
            const bool layer = p.layer_pre || p.layer_post;
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                float2 t[4];
                read(R{}, kY, warp_r, g, p.x, p.ld_x, yh[g]);
                read(T{}, kDh, warp_t, g, p.dh, p.ld_dh, t);
                read(T{}, kO, warp_t, g, p.o, p.ld_o, o[g]);
                if constexpr (gate_row) {
                    read(T{}, kG, warp_t, g, p.g, p.ld_g, a[g]);
                    gate_act8(p.gate, a[g]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    yh[g][i] = f2_mul(f2_add(yh[g][i], f2(-st.z)), f2(st.w));
                    sum[0][g][i] = f2_fma(t[i], yh[g][i], sum[0][g][i]);
                    if constexpr (kBias) sum[2][g][i] = f2_add(sum[2][g][i], t[i]);
                    t[i] = f2_mul(t[i], w[g][i]);
                    c1 = f2_fma(t[i], yh[g][i], c1);
                    dt[g][i] = f2_fma(t[i], f2(st.w), dt[g][i]);
                    o[g][i] = f2_mul(f2_add(o[g][i], f2(-st.x)), f2(st.y));
                    const float2 s = kIn == kPlain ? sw[g][i] : f2_mul(sw[g][i], a[g][i]), z = f2_mul(s, o[g][i]);
                    za = f2_fma(z, dt[g][i], za);
                    zy = f2_fma(z, yh[g][i], zy);
                    if (layer) {
                        c2 = f2_add(c2, t[i]);
                        z1 = f2_add(z1, z);
                        sa = f2_fma(s, dt[g][i], sa);
                        sy = f2_fma(s, yh[g][i], sy);
                        s1 = f2_add(s1, s);
                    }
                }
            }
            float2 means;
            if (layer) {
                float v[8] = {c1.x + c1.y, c2.x + c2.y, za.x + za.y, zy.x + zy.y, z1.x + z1.y, sa.x + sa.y, sy.x + sy.y, s1.x + s1.y};
                grp.template sums<8>(v);
                means = make_float2(-p.inv_c * v[0], p.layer_pre ? -p.inv_c * v[1] : 0.f);
                post_means = make_float2(fmaf(st.w, fmaf(means.x, v[3], means.y * v[4]), v[2]), p.layer_post ? fmaf(st.w, fmaf(means.x, v[6], means.y * v[7]), v[5]) : 0.f);
            } else {
                float v[4] = {c1.x + c1.y, za.x + za.y, zy.x + zy.y, 0.f};
                grp.template sums<4>(v);
                means = make_float2(-p.inv_c * v[0], 0.f);
                post_means = make_float2(fmaf(st.w * means.x, v[2], v[1]), 0.f);
            }
            post_means.x *= -p.inv_c; post_means.y *= -p.inv_c;
#pragma unroll
            for (int g = 0; g < kV; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) dt[g][i] = f2_fma(f2_fma(yh[g][i], f2(means.x), f2(means.y)), f2(st.w), dt[g][i]);
        } else if (p.has_pre) {
            float2 yh[kV][4], t[kV][4], c1 = f2(0.f), c2 = f2(0.f);
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                read(R{}, kY, warp_r, g, p.x, p.ld_x, yh[g]);
                read(T{}, kDh, warp_t, g, p.dh, p.ld_dh, t[g]);
                if constexpr (kWeightSlots) unpack8(slot_read<float, kThreads>(weight_slots + g * 2 * kThreads * 16), w[g]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    yh[g][i] = f2_mul(f2_add(yh[g][i], f2(-st.z)), f2(st.w));
                    sum[0][g][i] = f2_fma(t[g][i], yh[g][i], sum[0][g][i]);
                    if constexpr (kBias) sum[kBranch ? 2 : 1][g][i] = f2_add(sum[kBranch ? 2 : 1][g][i], t[g][i]);
                    t[g][i] = f2_mul(t[g][i], w[g][i]);
                    c1 = f2_fma(t[g][i], yh[g][i], c1);
                    c2 = f2_add(c2, t[g][i]);
                }
            }
            float2 means = p.layer_pre ? grp.sum<true>(c1.x + c1.y, c2.x + c2.y) : grp.sum<false>(c1.x + c1.y, 0.f);
            means.x *= -p.inv_c; means.y *= -p.inv_c;
#pragma unroll
            for (int g = 0; g < kV; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) dt[g][i] = f2_fma(f2_fma(yh[g][i], f2(means.x), f2_add(t[g][i], f2(means.y))), f2(st.w), dt[g][i]);
        }
#pragma unroll
        for (int g = 0; g < kV; ++g) {
            float2 dx[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) dx[i] = f2_mul(dt[g][i], f2(p.alpha));
            if (live) store8(static_cast<R *>(p.dx) + row * p.ld_dx, c[g], dx);
        }
        if constexpr (kBranch) {
            float2 u[kV][4], d1 = f2(0.f), d2 = f2(0.f);
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                if constexpr (!kOnce) {
                    read(T{}, kO, warp_t, g, p.o, p.ld_o, o[g]);
                    if constexpr (gate_row) read(T{}, kG, warp_t, g, p.g, p.ld_g, a[g]);
                }
                if constexpr (kWeightSlots) unpack8(slot_read<float, kThreads>(weight_slots + kWeights + g * 2 * kThreads * 16), sw[g]);
                if (!kOnce && p.has_post) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[g][i] = f2_mul(f2_add(o[g][i], f2(-st.x)), f2(st.y));
                }
                if constexpr (gate_row) {
                    float2 dg[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) dg[i] = f2_mul(dt[g][i], kBias ? f2_fma(o[g][i], sw[g][i], sb[g][i]) : f2_mul(o[g][i], sw[g][i]));
                    if (p.gate == 1) {
                        if constexpr (!kOnce) gate_act8(1, a[g]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dg[i] = f2_mul(dg[i], f2_mul(a[g][i], f2_fma(a[g][i], f2(-1.f), f2(1.f))));
                    }
                    if (live) store8(static_cast<T *>(p.dg) + row * p.ld_dg, c[g], dg);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 q = kIn == kPlain ? dt[g][i] : f2_mul(dt[g][i], a[g][i]), k = kIn == kShared ? dt[g][i] : q;
                    sum[1][g][i] = f2_fma(k, o[g][i], sum[1][g][i]);
                    if constexpr (kBias) sum[3][g][i] = f2_add(sum[3][g][i], k);
                    u[g][i] = f2_mul(q, sw[g][i]);
                    d1 = f2_fma(u[g][i], o[g][i], d1);
                    d2 = f2_add(d2, u[g][i]);
                }
            }
            if (kOnce || p.has_post) {
                float2 means = kOnce ? post_means : p.layer_post ? grp.sum<true>(d1.x + d1.y, d2.x + d2.y) : grp.sum<false>(d1.x + d1.y, 0.f);
                if constexpr (!kOnce) { means.x *= -p.inv_c; means.y *= -p.inv_c; }
#pragma unroll
                for (int g = 0; g < kV; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[g][i] = f2_mul(f2_fma(o[g][i], f2(means.x), f2_add(u[g][i], f2(means.y))), f2(st.y));
            }
#pragma unroll
            for (int g = 0; g < kV; ++g)
                if (live) store8(static_cast<T *>(p.d_o) + row * p.ld_do, c[g], u[g]);
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }

    // the block's sums: rows of a warp by shuffles, rows of different warps through shared memory
    ptx::copy_async_wait<0>();
    __syncthreads();
    float *all = reinterpret_cast<float *>(smem);                // [rows at a time][sum][group of columns][8 tpr]
    const int width = 8 * kV * p.tpr, slots_n = kThreads / max(p.tpr, 32), slot = p.tpr < 32 ? (int)(threadIdx.x >> 5) : mine;
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int j = 0; j < 8 * kV; ++j) {
            float v = (&sum[k][j / 8][j % 8 / 2].x)[j & 1];
            for (int o = p.tpr; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (p.tpr >= 32 || (int)(threadIdx.x & 31) < p.tpr) all[(slot * kSums + k) * width + j * p.tpr + lane] = v;
        }
    __syncthreads();
    float *out = p.part + (size_t)blockIdx.x * kSums * p.C;
    for (int i = threadIdx.x; i < kSums * width; i += kThreads) {
        float v = 0.f;
        for (int s = 0; s < slots_n; ++s) v += all[s * kSums * width + i];
        const int k = i / width, l = i % p.tpr, j = i % width / p.tpr;
        const Columns<kMove> cc(l, p.tpr, p.C, blockIdx.y * 8 * kV * kThreads + (j >> 3) * 8 * p.tpr);
        if (cc.has(j & 7)) out[(size_t)k * p.C + cc.at(j & 7)] = v;
    }
}

// ---------------------------------------------------------------- sums of the blocks' partial rows
struct BlockSums {
    const float *part;
    const void *g;                                         // the groups' gate rows, where they are shared
    void *dg;
    const float *scale, *w_post, *b_post;
    float *d_scale, *dw_post, *db_post, *dw_pre, *db_pre;
    long groups, ld_g, ld_dg;
    int chunks, C, sums, branch, bias, gate, grouped;
};
constexpr int kSumLanes = 32, kSumSlices = 32;

// A block has 32 columns and 32 slices of the partial rows (of a group's pieces where there are few groups, else of the groups), of the sums that
// go with the next norm (blockIdx.y = 0: dh y^, dh) or with the branch (1: Q, P).
template <typename T>
__global__ void __launch_bounds__(kSumLanes * kSumSlices) block_sums_kernel(BlockSums p) {
    __shared__ float2 sh[kSumSlices][kSumLanes];
    const int lane = threadIdx.x % kSumLanes, slice = threadIdx.x / kSumLanes, col = blockIdx.x * kSumLanes + lane;
    const bool branch = blockIdx.y == 1, yes = col < p.C;
    const int first = branch ? 1 : 0, second = (p.branch ? 2 : 1) + first;   // the two sums' places in a partial row
    int sub = kSumSlices;                                   // slices of one group
    while (sub > 1 && (long)(kSumSlices / sub) < p.groups) sub >>= 1;
    const int at_once = kSumSlices / sub, slot = slice / sub, part = slice % sub;
    ptx::grid_wait();
    const float s = yes && p.scale ? p.scale[col] : 1.f, w = yes && p.w_post ? p.w_post[col] : 1.f, b = yes && p.b_post ? p.b_post[col] : 0.f;
    float2 total = make_float2(0.f, 0.f);
    for (long g0 = 0; g0 < p.groups; g0 += at_once) {
        const long grp = g0 + slot;
        float2 v = make_float2(0.f, 0.f);
        if (yes && grp < p.groups) {
            const float *src = p.part + ((size_t)grp * p.chunks * p.sums + first) * p.C + col;
            const size_t row = (size_t)p.sums * p.C, other = (size_t)(second - first) * p.C;
            if (p.bias) {
#pragma unroll 8
                for (int ch = part; ch < p.chunks; ch += sub) {
                    v.x += src[ch * row];
                    v.y += src[ch * row + other];
                }
            } else {
#pragma unroll 8
                for (int ch = part; ch < p.chunks; ch += sub) v.x += src[ch * row];
            }
        }
        if (p.grouped && branch) {
            // the group's own sums: one thread per column puts the slices together
            if (sub > 1) {
                sh[slice][lane] = v;
                __syncthreads();
                if (part == 0)
                    for (int q = 1; q < sub; ++q) v = f2_add(v, sh[slice + q][lane]);
                __syncthreads();
            }
            if (part == 0 && yes && grp < p.groups) {
                const float g = to_f32(static_cast<const T *>(p.g)[grp * p.ld_g + col]), a = gate_act(p.gate, g);
                const float slope = p.gate == 1 ? a * (1.f - a) : 1.f;
                from_f32(static_cast<T *>(p.dg)[grp * p.ld_dg + col], s * slope * fmaf(w, v.x, b * v.y));
                v = f2_mul(v, f2(a));
            } else {
                v = make_float2(0.f, 0.f);
            }
        }
        total = f2_add(total, v);
    }
    sh[slice][lane] = total;
    __syncthreads();
    for (int half = kSumSlices / 2; half > 1; half >>= 1) {
        if (slice < half) sh[slice][lane] = f2_add(sh[slice][lane], sh[slice + half][lane]);
        __syncthreads();
    }
    if (slice != 0 || !yes) return;
    total = f2_add(sh[0][lane], sh[1][lane]);
    if (!branch) {
        if (p.dw_pre) p.dw_pre[col] = total.x;
        if (p.db_pre) p.db_pre[col] = total.y;
    } else {
        if (p.d_scale) p.d_scale[col] = fmaf(w, total.x, b * total.y);
        if (p.dw_post) p.dw_post[col] = s * total.x;
        if (p.db_post) p.db_post[col] = s * total.y;
    }
}

}  // namespace flare
