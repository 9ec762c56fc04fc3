// Tokens on their way into a model: embedding lookup and its gradient, and dropout.
//
//     embed     y[n] = drop(scale E[t_n] + P[n mod L])             dE[v] = scale sum_{t_n = v} drop'(dy[n]),  dP[l] = sum_{n mod L = l} drop'(dy[n])
//     dropout   y = residual + drop(x)                              dx = drop'(dy)
//
// drop multiplies an element by 0 or by keep = 65536 / (65536 - thr), drop' = drop with the same factors.  Which, says a counter-based generator,
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011): its counter is (column / 8, row, offset), its key the seed, and of its 128 bits every one of the eight
// columns takes 16: kept where they are at least thr = round(65536 p).  So the mask is a function of where an element stands, nothing of it is stored, and a
// backward pass forms it again.  Eight columns a call are what makes it cheap beside the memory traffic: ten rounds are 20 wide multiplications and 20
// three-way exclusive ors, 5 a column, where a column of two bytes in and two out has some 22 issue slots before memory is no longer the bound; 32 bits a
// column would take twice that for a p that is exact to 2^-33 instead of 2^-17 (the factor that makes up for the dropped is that of the p used, so that the mean is kept).
//
// All of it is bound by memory: one pass, 16 bytes a load, a thread eight columns of a row.
#pragma once

#include "flare_common.cuh"
#include "flare_ptx.cuh"

namespace flare {

// Generator and threshold; thr = 0: nothing is dropped.  The rounds' keys (key + r times two odd constants) are the same for all: they come from the host, as operands out of constant memory.
struct DropArgs {
    uint32_t thr;
    float keep;
    uint32_t k0[10], k1[10];
    uint64_t offset;
    const int64_t *step;                                      // device, or null: added to offset
    __device__ __forceinline__ uint32_t below() const { return (thr << 16) - 1; }   // the largest word whose high half is below thr (thr is 1 to 65536)
};
struct DropKey { uint32_t c2, c3; };                          // the counter's upper words
__device__ __forceinline__ DropKey drop_key(const DropArgs &d) {
    const uint64_t at = d.offset + (d.thr != 0 && d.step != nullptr ? (uint64_t)*d.step : 0ull);
    return DropKey{(uint32_t)at, (uint32_t)(at >> 32)};
}
__device__ __forceinline__ uint4 philox(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row) {
    uint32_t c0 = group, c1 = row, c2 = k.c2, c3 = k.c3;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ d.k0[r];
        c2 = (uint32_t)(a >> 32) ^ c3 ^ d.k1[r];
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Eight columns' values through dropout: what is dropped is 0 whatever it was.
__device__ __forceinline__ void drop8(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row, float (&v)[8]) {
    const uint4 u = philox(d, k, group, row);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (w[i] & 0xffffu) >= d.thr ? v[2 * i] * d.keep : 0.f;
        v[2 * i + 1] = w[i] > d.below() ? v[2 * i + 1] * d.keep : 0.f;    // (the high half is at least thr)
    }
}
// Zeros where they are dropped, no factor.
__device__ __forceinline__ void zero8(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row, float (&v)[8]) {
    const uint4 u = philox(d, k, group, row);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (w[i] & 0xffffu) >= d.thr ? v[2 * i] : 0.f;
        v[2 * i + 1] = w[i] > d.below() ? v[2 * i + 1] : 0.f;
    }
}
// What is kept of eight columns' values, added up without the factor.
__device__ __forceinline__ void add_kept8(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row, const float (&v)[8], float (&sum)[8]) {
    const uint4 u = philox(d, k, group, row);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0xffffu) >= d.thr) sum[2 * i] += v[2 * i];
        if (w[i] > d.below()) sum[2 * i + 1] += v[2 * i + 1];
    }
}
// The same as eight bits.
__device__ __forceinline__ uint32_t keep8(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row) {
    const uint4 u = philox(d, k, group, row);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= ((w[i] & 0xffffu) >= d.thr ? 1u : 0u) << (2 * i);
        bits |= (w[i] >> 16 >= d.thr ? 1u : 0u) << (2 * i + 1);
    }
    return bits;
}

// Where a row begins, of rows ld elements apart.
__device__ __forceinline__ size_t row_at(uint32_t row, uint32_t ld) { return (uint64_t)row * ld; }

// Eight neighbouring elements, as they lie in memory (rows on 16-byte boundaries) and as floats.
template <typename T> struct Eight { uint4 q[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ void load8(const T *p, Eight<T> &e) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.q[i] = reinterpret_cast<const uint4 *>(p)[i];
}
template <typename T> __device__ __forceinline__ void floats8(const Eight<T> &e, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(reinterpret_cast<const T *>(e.q)[i]);
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    __align__(16) T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) from_f32(e[i], v[i]);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(e)[i];
}

// A thread's walk over the groups of columns of all rows, `step` groups at a time, without divisions.
struct GroupWalk {
    uint32_t row, group, drow, dgroup, groups;
    __device__ __forceinline__ GroupWalk(uint64_t first, uint64_t step, uint32_t groups_) : groups(groups_) {
        row = (uint32_t)(first / groups); group = (uint32_t)(first % groups);
        drow = (uint32_t)(step / groups); dgroup = (uint32_t)(step % groups);
    }
    __device__ __forceinline__ bool next() {                  // (whether a group more made a row more)
        row += drow; group += dgroup;
        const bool over = group >= groups;
        if (over) { group -= groups; ++row; }
        return over;
    }
};
// And over positions, row mod L.
struct PositionWalk : GroupWalk {
    uint32_t at, dat, L;
    __device__ __forceinline__ PositionWalk(uint64_t first, uint64_t step, uint32_t groups_, uint32_t L_) : GroupWalk(first, step, groups_), L(L_) {
        at = row % L; dat = drow % L;
    }
    __device__ __forceinline__ void next() {
        at += dat + (GroupWalk::next() ? 1 : 0);
        if (at >= L) at -= L;
    }
};

// ---------------------------------------------------------------- dropout
struct DropoutArgs {
    const void *x, *residual;                                 // residual: null if there is none
    void *y;
    uint32_t ld_x, ld_r, ld_y, rows, C;
    DropArgs drop;
};
constexpr int kTokenThreads = 256;

// X: type of what goes through dropout, R: of the residual and the result.  Backward: no residual, X the gradient's type, R that of dx.
// kVec: rows of 8 m columns on 16-byte boundaries.  Else a warp takes 256 columns of a row, neighbouring lanes neighbouring columns: lane l forms the
// bits of the columns 8 l .. 8 l + 7 and the others ask it for theirs.
template <typename X, typename R, bool kVec>
__global__ void __launch_bounds__(kTokenThreads) dropout_kernel(const DropoutArgs a) {
    ptx::grid_launch();
    ptx::grid_wait();
    const X *x = static_cast<const X *>(a.x);
    const R *res = static_cast<const R *>(a.residual);
    R *y = static_cast<R *>(a.y);
    const DropKey key = drop_key(a.drop);
    if constexpr (kVec) {
        constexpr int kBatch = 4;
        GroupWalk w((uint64_t)blockIdx.x * kTokenThreads + threadIdx.x, (uint64_t)gridDim.x * kTokenThreads, a.C / 8);
        while (w.row < a.rows) {
            uint32_t row[kBatch], group[kBatch];
            Eight<X> e[kBatch];
            Eight<R> f[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                row[k] = w.row; group[k] = w.group;
                if (w.row < a.rows) {
                    load8(x + row_at(w.row, a.ld_x) + w.group * 8, e[k]);
                    if (res) load8(res + row_at(w.row, a.ld_r) + w.group * 8, f[k]);
                }
                w.next();
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (row[k] >= a.rows) break;
                float v[8];
                floats8(e[k], v);
                if (a.drop.thr) drop8(a.drop, key, group[k], row[k], v);
                if (res) {
                    float r[8];
                    floats8(f[k], r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += r[i];
                }
                store8(y + row_at(row[k], a.ld_y) + group[k] * 8, v);
            }
        }
    } else {
        const uint32_t lane = threadIdx.x & 31, warps = kTokenThreads / 32;
        GroupWalk w((uint64_t)blockIdx.x * warps + (threadIdx.x >> 5), (uint64_t)gridDim.x * warps, (a.C + 255) / 256);
        for (; w.row < a.rows; w.next()) {
            const uint32_t c0 = w.group * 256 + lane;
            const X *px = x + row_at(w.row, a.ld_x) + c0;
            const R *pr = res ? res + row_at(w.row, a.ld_r) + c0 : nullptr;
            R *py = y + row_at(w.row, a.ld_y) + c0;
            float v[8], r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = c0 + 32 * k < a.C ? to_f32(px[32 * k]) : 0.f;
                r[k] = pr && c0 + 32 * k < a.C ? to_f32(pr[32 * k]) : 0.f;
            }
            const uint32_t bits = a.drop.thr ? keep8(a.drop, key, w.group * 32 + lane, w.row) : 0xffu;
            const float keep = a.drop.thr ? a.drop.keep : 1.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t b = __shfl_sync(0xffffffffu, bits, 4 * k + (lane >> 3));
                const float d = b >> (lane & 7) & 1 ? v[k] * keep : 0.f;
                if (c0 + 32 * k < a.C) from_f32(py[32 * k], pr ? d + r[k] : d);
            }
        }
    }
}

// Contiguous rows whose width eight does not divide: moved 16 bytes at a time all the same, as one long row.  A block has rows that begin on an eighth element (a multiple of eight of them),
// forms their bits, a call of the generator a group of a row's columns, and lays them in shared memory bit by bit, where eight elements find theirs as one byte.  40028 x 333 in float16
// (53 MB): 28 us with neighbouring lanes on neighbouring columns, above; 18.1 (2.9 TB/s) this way, bound by instructions.
struct DropoutFlat {
    DropoutArgs a;
    uint32_t tile_rows;
};
template <typename X, typename R>
__global__ void __launch_bounds__(kTokenThreads) dropout_flat_kernel(const DropoutFlat f) {
    extern __shared__ uint32_t bits[];
    ptx::grid_launch();
    ptx::grid_wait();
    const DropoutArgs &a = f.a;
    const DropKey key = drop_key(a.drop);
    const uint32_t row0 = blockIdx.x * f.tile_rows, rows = min(f.tile_rows, a.rows - row0), elements = rows * a.C, words = (elements + 31) / 32;
    const X *x = static_cast<const X *>(a.x) + row_at(row0, a.C);
    const R *res = a.residual ? static_cast<const R *>(a.residual) + row_at(row0, a.C) : nullptr;
    R *y = static_cast<R *>(a.y) + row_at(row0, a.C);
    constexpr int kBatch = 2;
    Eight<X> e[kBatch];
    Eight<R> r[kBatch];
    auto ask = [&](uint32_t i0) {                             // (the first of them before the bits are formed)
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const uint32_t i = (i0 + k * kTokenThreads) * 8;
            if (i + 8 <= elements) {
                load8(x + i, e[k]);
                if (res) load8(res + i, r[k]);
            }
        }
    };
    ask(threadIdx.x);
    for (uint32_t i = threadIdx.x; i < words; i += kTokenThreads) bits[i] = 0;
    __syncthreads();
    for (GroupWalk w(threadIdx.x, kTokenThreads, (a.C + 7) / 8); w.row < rows; w.next()) {
        const uint32_t at = w.row * a.C + w.group * 8, n = min(8u, a.C - w.group * 8);
        const uint64_t b = (uint64_t)(keep8(a.drop, key, w.group, row0 + w.row) & ((1u << n) - 1)) << (at & 31);
        atomicOr(bits + (at >> 5), (uint32_t)b);
        if (b >> 32) atomicOr(bits + (at >> 5) + 1, (uint32_t)(b >> 32));
    }
    __syncthreads();
    for (uint32_t i0 = threadIdx.x; i0 * 8 < elements; i0 += kBatch * kTokenThreads) {
        if (i0 != threadIdx.x) ask(i0);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const uint32_t i = (i0 + k * kTokenThreads) * 8;
            if (i >= elements) break;
            const uint32_t b = bits[i >> 5] >> (i & 31);
            if (i + 8 <= elements) {
                float v[8];
                floats8(e[k], v);
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] = b >> c & 1 ? v[c] * a.drop.keep : 0.f;
                if (res) {
                    float u[8];
                    floats8(r[k], u);
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] += u[c];
                }
                store8(y + i, v);
            } else {                                          // the last few of all
                for (uint32_t c = 0; i + c < elements; ++c) {
                    const float d = b >> c & 1 ? to_f32(x[i + c]) * a.drop.keep : 0.f;
                    from_f32(y[i + c], res ? d + to_f32(res[i + c]) : d);
                }
            }
        }
    }
}

// ---------------------------------------------------------------- embedding, forward
struct EmbedArgs {
    const void *tokens, *table, *positions;                   // positions: null if there are none
    void *y;
    uint32_t ld_t, ld_y, rows, C, L;                          // L: positions, row n takes n mod L
    uint32_t vocab;
    float scale;
    DropArgs drop;
    int wide;                                                 // tokens are 64 bits
};
// A token, or ~0 for one that has no row.
__device__ __forceinline__ uint32_t token_at(const void *tokens, int wide, uint32_t n, uint32_t vocab) {
    if (!wide) {
        const uint32_t t = static_cast<const uint32_t *>(tokens)[n];
        return t < vocab ? t : ~0u;
    }
    const uint2 t = static_cast<const uint2 *>(tokens)[n];
    return t.y == 0 && t.x < vocab ? t.x : ~0u;
}
// T: type of the tables, O: of the rows.  kWidth: groups of eight columns next to each other that a thread takes (two share a row's token and addresses: 260 instructions a group became 189 with positions and dropout, which is what bounds it: 131072 rows of 128 over 256 words take 17.3 us, 3.1 TB/s of rows read and written), 0: rows
// off 16-byte boundaries.
template <typename T, typename O, int kWidth>
__global__ void __launch_bounds__(kTokenThreads, kWidth == 2 && sizeof(T) + sizeof(O) > 4 ? 3 : 4) embed_kernel(const EmbedArgs a) {
    ptx::grid_launch();
    ptx::grid_wait();
    const T *table = static_cast<const T *>(a.table), *pos = static_cast<const T *>(a.positions);
    O *y = static_cast<O *>(a.y);
    const DropKey key = drop_key(a.drop);
    if constexpr (kWidth > 0) {
        const float scale = a.scale * a.drop.keep;
        constexpr int kBatch = 2 / kWidth;
        PositionWalk w((uint64_t)blockIdx.x * kTokenThreads + threadIdx.x, (uint64_t)gridDim.x * kTokenThreads, a.C / (8 * kWidth), a.L);
        while (w.row < a.rows) {
            uint32_t row[kBatch], col[kBatch], t[kBatch];
            Eight<T> e[kBatch][kWidth], f[kBatch][kWidth];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                row[k] = w.row; col[k] = w.group * (8 * kWidth);
                t[k] = ~0u;
                if (w.row < a.rows) {
                    t[k] = token_at(a.tokens, a.wide, w.row, a.vocab);
                    if (pos)
#pragma unroll
                        for (int i = 0; i < kWidth; ++i) load8(pos + row_at(w.at, a.C) + col[k] + 8 * i, f[k][i]);
                }
                w.next();
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (t[k] != ~0u)
#pragma unroll
                    for (int i = 0; i < kWidth; ++i) load8(table + row_at(t[k], a.ld_t) + col[k] + 8 * i, e[k][i]);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (row[k] >= a.rows) break;
                O *out = y + row_at(row[k], a.ld_y) + col[k];
#pragma unroll
                for (int i = 0; i < kWidth; ++i) {
                    float v[8] = {};
                    if (pos) {
                        floats8(f[k][i], v);
#pragma unroll
                        for (int c = 0; c < 8; ++c) v[c] *= a.drop.keep;
                    }
                    if (t[k] != ~0u) {
                        float r[8];
                        floats8(e[k][i], r);
#pragma unroll
                        for (int c = 0; c < 8; ++c) v[c] = fmaf(r[c], scale, v[c]);
                    }
                    if (a.drop.thr) zero8(a.drop, key, col[k] / 8 + i, row[k], v);
                    store8(out + 8 * i, v);
                }
            }
        }
    } else {
        const uint32_t lane = threadIdx.x & 31, warps = kTokenThreads / 32;
        GroupWalk w((uint64_t)blockIdx.x * warps + (threadIdx.x >> 5), (uint64_t)gridDim.x * warps, (a.C + 255) / 256);
        for (; w.row < a.rows; w.next()) {
            const uint32_t c0 = w.group * 256 + lane;
            const uint32_t t = token_at(a.tokens, a.wide, w.row, a.vocab);
            const bool there = t != ~0u;
            const float keep = a.drop.keep, scale = a.scale * keep;
            const T *pe = table + (there ? row_at(t, a.ld_t) + c0 : 0), *pp = pos ? pos + row_at(w.row % a.L, a.C) + c0 : nullptr;
            O *py = y + row_at(w.row, a.ld_y) + c0;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool in = c0 + 32 * k < a.C;
                v[k] = pp && in ? to_f32(pp[32 * k]) * keep : 0.f;
                if (there && in) v[k] = fmaf(to_f32(pe[32 * k]), scale, v[k]);
            }
            const uint32_t bits = a.drop.thr ? keep8(a.drop, key, w.group * 32 + lane, w.row) : 0xffu;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t b = __shfl_sync(0xffffffffu, bits, 4 * k + (lane >> 3));
                const float d = b >> (lane & 7) & 1 ? v[k] : 0.f;
                if (c0 + 32 * k < a.C) from_f32(py[32 * k], d);
            }
        }
    }
}

// ---------------------------------------------------------------- embedding, backward
//
// Rows that met the same token are added up in the order of the rows, whatever else the GPU does: the tokens are sorted (stably), the sorted rows are cut
// into chunks of the same length, and a thread adds up eight columns of a chunk's rows.  A token all of whose rows lie in one chunk is finished there; chunks of one block are
// joined in shared memory, and what reaches over the end of a block's rows leaves float32 sums, which a second kernel adds up in their order.  So a token that every third row has
// takes no longer than rare ones, and no sum depends on the order in which blocks run.
//
// Positions are the same with an order that need not be sorted: row i of it is row (i mod B) L + i / B of the batch, its "token" i / B.
//
// The sort: one cluster of blocks (up to 16 of 1024 threads), each a stretch of the tokens, each of its warps a stretch of that.  A pass over a digit of up to
// ten bits: every warp counts its stretch, the counts before it are added up over the warps in shared memory and over the blocks through distributed shared memory, and
// every warp puts its tokens where those say (lanes with the same digit find one another by a ballot a bit): in shared memory first, so that what goes to memory are stretches of
// neighbours (up to kSortStaged tokens a block, 64 KB beside the counts of ten bits; beyond that as they come: gradients of 131072 tokens of 16 columns over 256 words take 33.4 us, of 132000 33.9, over 32000 words 60.0 and 60.8).  One launch, two barriers of the cluster a pass, where kernels of a count, a scan and a scatter each would be three launches a
// pass: 17 us for 131072 tokens in one pass and for 16396 in two, by latency.
constexpr int kSortThreads = 1024, kSortBits = 10, kSortBatch = 4, kSortBlocks = 16;
constexpr uint32_t kSortStaged = 8192;
struct SortArgs {
    const void *tokens;
    int wide;
    uint32_t rows, vocab;
    int passes, bits;                                         // digits of the key (a token in range, or vocab for one that is not)
    uint2 *pairs[2];                                          // key, row; pass p writes to [p & 1]
    int staged;                                               // a block's stretch fits shared memory: it is sorted there first
};
__host__ __device__ __forceinline__ int sorted_in(int passes) { return (passes - 1) & 1; }
namespace ptx {
__device__ __forceinline__ uint32_t lds_cluster(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t v;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(v));
    return v;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t v;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(v));
    return v;
}
}  // namespace ptx
// Lanes with the same digit (up to kSortBits bits), of those that take part.  (By ballots: match.any took a quarter longer.)
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, uint32_t taking) {
    uint32_t same = taking;
#pragma unroll
    for (int b = 0; b < kSortBits; ++b) {
        const int set = (int)(digit << (31 - b));
        same &= ~(__ballot_sync(0xffffffffu, set < 0) ^ (uint32_t)(set >> 31));
    }
    return same;
}

// Sums over the threads before this one, of two numbers; all threads.
__device__ __forceinline__ uint2 before_in_block(uint2 own, uint2 *scan) {
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto over_lanes = [&](uint2 s) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, s.x, o), y = __shfl_up_sync(0xffffffffu, s.y, o);
            if (lane >= (uint32_t)o) { s.x += x; s.y += y; }
        }
        return s;
    };
    const uint2 sum = over_lanes(own);
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    if (warp == 0) scan[lane] = over_lanes(scan[lane]);
    __syncthreads();
    const uint2 ahead = warp > 0 ? scan[warp - 1] : make_uint2(0, 0);
    return make_uint2(sum.x - own.x + ahead.x, sum.y - own.y + ahead.y);
}
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const SortArgs a) {
    extern __shared__ __align__(16) uint32_t counts[];        // [32 warps][bins], [bins] of the block, [bins] from places here to places in memory, [32] pairs of a scan, pairs
    ptx::grid_wait();                                         // (then the launch behind this one: positions, which wait for nothing of this one's, but for what came before it)
    __threadfence();                                          // (SumArgs::beside_zero)
    ptx::grid_launch();
    const uint32_t blocks = ptx::cluster_size(), rank = ptx::cluster_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // stretches: of a block, of a warp (whole groups of 32)
    const uint32_t per_warp = ((a.rows + blocks * 32 - 1) / (blocks * 32) + 31) / 32 * 32;
    auto clip = [&](uint64_t i) { return (uint32_t)min(i, (uint64_t)a.rows); };
    const uint32_t first = clip((uint64_t)(rank * 32 + warp) * per_warp), last = clip((uint64_t)(rank * 32 + warp + 1) * per_warp);
    const uint32_t own = clip((uint64_t)(rank + 1) * 32 * per_warp) - clip((uint64_t)rank * 32 * per_warp);   // of the block
    const uint32_t bins = 1u << a.bits;
    uint32_t *mine = counts + warp * bins, *block = counts + 32 * bins, *shift_of = block + bins;
    uint2 *scan = reinterpret_cast<uint2 *>(shift_of + bins), *stage = scan + 32;
    for (int pass = 0; pass < a.passes; ++pass) {
        const uint32_t shift = pass * a.bits;
        const uint2 *in = a.pairs[(pass & 1) ^ 1];
        uint2 *out = a.pairs[pass & 1];
        auto pair_of = [&](uint32_t i) -> uint2 {
            if (pass > 0) return __ldcg(in + i);
            return make_uint2(min(token_at(a.tokens, a.wide, i, a.vocab), a.vocab), i);
        };
        for (uint32_t i = threadIdx.x; i < 8 * bins; i += kSortThreads) reinterpret_cast<uint4 *>(counts)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        // (kSortBatch groups of 32 are asked for before the first is looked at)
        for (uint32_t i0 = first; i0 < last; i0 += 32 * kSortBatch) {
            uint32_t digit[kSortBatch];
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) digit[j] = i0 + 32 * j + lane < last ? pair_of(i0 + 32 * j + lane).x >> shift & (bins - 1) : ~0u;
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j)
                if (digit[j] != ~0u) atomicAdd(mine + digit[j], 1u);
        }
        __syncthreads();
        // before each warp within the block
        const uint32_t d = threadIdx.x;
        uint32_t total = 0;
        if (d < bins) {
#pragma unroll 8
            for (uint32_t w = 0; w < 32; ++w) {
                const uint32_t c = counts[w * bins + d];
                counts[w * bins + d] = total;
                total += c;
            }
            block[d] = total;
        }
        ptx::cluster_meet();
        // before this block, and of all blocks
        uint32_t before = 0, all = 0;
        if (d < bins) {
            uint32_t c[kSortBlocks];
#pragma unroll
            for (uint32_t r = 0; r < kSortBlocks; ++r) c[r] = r < blocks ? ptx::lds_cluster(ptx::in_block(ptx::smem_u32(block + d), r)) : 0u;
#pragma unroll
            for (uint32_t r = 0; r < kSortBlocks; ++r) {
                if (r < rank) before += c[r];
                all += c[r];
            }
        }
        // before each digit: of all, and of this block's
        const uint2 ahead = before_in_block(make_uint2(all, total), scan);
        const uint32_t global = ahead.x + before, base = a.staged ? ahead.y : global;
        if (d < bins) {
            shift_of[d] = global - base;
#pragma unroll 8
            for (uint32_t w = 0; w < 32; ++w) counts[w * bins + d] += base;
        }
        __syncthreads();
        for (uint32_t i0 = first; i0 < last; i0 += 32 * kSortBatch) {
            uint2 pair[kSortBatch];
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) pair[j] = i0 + 32 * j + lane < last ? pair_of(i0 + 32 * j + lane) : make_uint2(0, 0);
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                if (i0 + 32 * j >= last) break;
                const bool in_range = i0 + 32 * j + lane < last;
                const uint32_t digit = pair[j].x >> shift & (bins - 1);
                const uint32_t same = same_digit(digit, __ballot_sync(0xffffffffu, in_range)), lower = same & ((1u << lane) - 1);
                uint32_t at = 0;
                if (in_range) at = mine[digit] + __popc(lower);
                __syncwarp();
                if (in_range) {
                    if (lower == 0) mine[digit] += __popc(same);
                    (a.staged ? stage : out)[at] = pair[j];
                }
                __syncwarp();
            }
        }
        if (a.staged) {
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < own; i += kSortThreads) {
                const uint2 pair = stage[i];
                out[i + shift_of[pair.x >> shift & (bins - 1)]] = pair;
            }
        }
        // (what was put into memory is seen by all blocks; nobody's counts are read any more)
        ptx::cluster_meet();
    }
}

// Rows of the gradient that no token has met: zeros.  A lane looks one row up among the sorted tokens, a warp writes what 32 of them want.  The launch behind it (the sums; of a large table half is left to be
// done beside the joins) need not wait for this, only for the one before it, which has ended when every block here has got past its wait, and runs beside it; its last block then waits, so that what comes
// behind both comes behind this too.  16396 tokens over 50021 rows of 1000, whose 200 MB take 29 us on their own: 87 us one after the other, 83 with all of it beside the sums, 73 to 78 so.
constexpr int kZeroThreads = 128;
struct ZeroArgs {
    const uint2 *pairs;
    uint32_t items, vocab, first, last;                       // groups of 32 rows, from first to before last
    uint64_t row_bytes;
    uint8_t *out;
};
template <typename T>                                         // of an element's size
__device__ __forceinline__ void zero_bytes(uint8_t *p, uint64_t n) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t head = min(n, (uint64_t)(-reinterpret_cast<uintptr_t>(p) & 15u)), body = (n - head) / 16, tail = n - head - body * 16;
    if (lane * sizeof(T) < head) reinterpret_cast<T *>(p)[lane] = 0;
    uint4 *q = reinterpret_cast<uint4 *>(p + head);
#pragma unroll 4
    for (uint64_t i = lane; i < body; i += 32) q[i] = make_uint4(0, 0, 0, 0);
    if (lane * sizeof(T) < tail) reinterpret_cast<T *>(q + body)[lane] = 0;
}
template <typename T>
__global__ void __launch_bounds__(kZeroThreads) embed_zero_kernel(const ZeroArgs a) {
    ptx::grid_wait();
    __threadfence();                                          // (SumArgs::beside_zero)
    ptx::grid_launch();
    const uint32_t warps = gridDim.x * (kZeroThreads / 32), lane = threadIdx.x & 31;
    for (uint32_t g = a.first + blockIdx.x * (kZeroThreads / 32) + (threadIdx.x >> 5); g < a.last; g += warps) {
        const uint32_t row = g * 32 + lane;
        uint32_t lo = 0, hi = a.items;                        // the first sorted token that is not below the row
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (a.pairs[mid].x < row) lo = mid + 1;
            else hi = mid;
        }
        const bool none = row < a.vocab && (lo == a.items || a.pairs[lo].x != row);
        uint32_t m = __ballot_sync(0xffffffffu, none);
        while (m != 0) {                                      // rows next to each other at once
            const uint32_t from = __ffs(m) - 1, rest = ~(m >> from), n = rest == 0 ? 32 : __ffs(rest) - 1;
            zero_bytes<T>(a.out + (uint64_t)(g * 32 + from) * a.row_bytes, n * a.row_bytes);
            m &= n + from >= 32 ? (1u << from) - 1 : ~(((1u << n) - 1) << from);
        }
    }
}

// Sums over runs of equal keys.  Two tasks in one launch: tokens, and positions.
struct SumTask {
    const uint2 *pairs;                                       // sorted: key, row; null: positions
    uint32_t items, batch, L;                                 // items of the order; positions: batch items, rows of an item
    uint32_t most;                                            // keys from here on are none
    void *out;
    float scale;
    int add;                                                  // to what is there
    float *part;                                              // [blocks along the order][2][columns]: of the run a block's rows begin with, of the one they end with
    uint32_t T, spans;                                        // rows of a chunk; blocks along the order, of SumArgs::chunks chunks each
};
struct SumArgs {
    SumTask task[2];
    const void *dy;
    uint32_t ld_dy, C, columns;                               // columns: C up to whole groups of eight
    // Launches that need not wait for the one before them (embed_zero_kernel; of positions: the sort): 1: the sums, 2: the joins too.  They begin when all blocks of that one have got past their wait for what these
    // need too.  A wait makes what came before visible to the grid that waits; to these it is made so by fences on both sides: of the grid between before it lets them begin, and of theirs before they read.
    int beside_zero;
    uint32_t threads, lanes, tiles, chunks;                   // threads of a block; side by side over a row's units of columns, blocks side by side, chunks of a block one after the other
    DropArgs drop;
};
__device__ __forceinline__ uint32_t key_at(const SumTask &t, uint32_t i) { return t.pairs ? t.pairs[i].x : i / t.batch; }
// Walks over the order's (key, row).
struct OrderWalk {
    const SumTask &t;
    uint32_t i, l, b;
    __device__ __forceinline__ OrderWalk(const SumTask &t_, uint32_t i_) : t(t_), i(i_), l(0), b(0) {
        if (!t.pairs) { l = i / t.batch; b = i - l * t.batch; }
    }
    __device__ __forceinline__ uint2 next(uint32_t end) {
        if (i >= end) return make_uint2(~0u, 0u);
        if (t.pairs) return t.pairs[i++];
        const uint2 r = make_uint2(l, b * t.L + l);
        ++i;
        if (++b == t.batch) { b = 0; ++l; }
        return r;
    }
};
// kVec: dy's and out's rows on 16-byte boundaries and C a multiple of 8.
template <typename O, bool kVec>
__device__ __forceinline__ void sum_load(const SumArgs &a, const O *dy, uint32_t row, uint32_t group, Eight<O> &e) {
    const O *p = dy + row_at(row, a.ld_dy) + group * 8;
    if constexpr (kVec) load8(p, e);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (group * 8 + i < a.C) reinterpret_cast<O *>(e.q)[i] = p[i];
            else from_f32(reinterpret_cast<O *>(e.q)[i], 0.f);
    }
}
template <typename T, bool kVec>
__device__ __forceinline__ void sum_store(const SumTask &t, uint32_t C, uint32_t key, uint32_t group, const float (&v)[8]) {
    T *p = static_cast<T *>(t.out) + row_at(key, C) + group * 8;
    if constexpr (kVec) {
        float r[8] = {};
        if (t.add) {
            Eight<T> e;
            load8(p, e);
            floats8(e, r);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = fmaf(v[i], t.scale, r[i]);
        store8(p, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (group * 8 + i < C) from_f32(p[i], fmaf(v[i], t.scale, t.add ? to_f32(p[i]) : 0.f));
    }
}
__device__ __forceinline__ void put8(float *to, const float (&v)[8]) {
    reinterpret_cast<float4 *>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void add8(float (&v)[8], const float *from) {
    const float4 x = reinterpret_cast<const float4 *>(from)[0], y = reinterpret_cast<const float4 *>(from)[1];
    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
}
enum { kRunOpen = 1, kRunGoesOn = 2, kRunThrough = 4 };       // a chunk's first run began before it; its last one goes on behind it; the two are the same and all of it
// Blocks of 128 threads where a row takes up to 16 of them, so that no SM waits for the last of few large ones, else of 256, where a block joins more chunks by itself (131072 rows of 256 over 32000 words: 84 us with
// blocks of 64, 80 with 128 or 256; 65536 of 512: 92, 78, 74).  Chunks are 16 rows, longer where there is more to do: 16384 rows of 4096 take 186 us in chunks of 16, 144 of 64; 65536 of 512 over 256 words take 50.3 of 16,
// 44.6 of 28; 131072 of 128 over 32000 take 65.6 of 16, 79.5 of 32.  It is bound by instructions: 32 x 4096 rows of 128 over 256 words with positions take 42 to 45 us in all, 17 to 20 of them the sort.
constexpr int kSumThreads = 256;
__host__ __device__ constexpr size_t sum_smem(uint32_t threads, int width) { return threads * (size_t)(2 * 32 * width + 8); }
// kWidth: groups of eight columns next to each other that a thread adds up (two share what there is to know of a row: 167 instructions a group and row became 108; of 1024 columns 50.5 us against 54.7 for 16384 rows, but of 128 columns 72 against 64 for 131072: rows need 32 such threads), 0: one, off 16-byte boundaries.
template <typename O, typename T, int kWidth>
__global__ void __launch_bounds__(kSumThreads, sizeof(O) == 4 || kWidth == 2 ? 2 : 3) embed_sum_kernel(const SumArgs a) {
    constexpr int kW = kWidth == 2 ? 2 : 1;
    constexpr bool kVec = kWidth > 0;
    extern __shared__ __align__(16) float first_sum[];        // [threads][8 kW], and the same of last runs; by chunk: key of the first run, flags
    float *last_sum = first_sum + blockDim.x * 8 * kW;
    uint32_t *first_run = reinterpret_cast<uint32_t *>(last_sum + blockDim.x * 8 * kW), *flags = first_run + blockDim.x;
    if (a.beside_zero) {
        __threadfence();
    } else {
        ptx::grid_launch();
        ptx::grid_wait();
    }
    const bool second = blockIdx.x < a.task[1].spans * a.tiles;           // (positions first: their chunks are the longer ones)
    const SumTask &t = a.task[second];
    const uint32_t at = blockIdx.x - (second ? 0 : a.task[1].spans * a.tiles), span = at / a.tiles, k = threadIdx.x / a.lanes;
    const uint32_t group = ((at - span * a.tiles) * a.lanes + threadIdx.x - k * a.lanes) * kW, groups = a.columns / 8;
    const uint64_t i0_64 = ((uint64_t)span * a.chunks + k) * t.T;
    const uint32_t i0 = (uint32_t)min(i0_64, (uint64_t)t.items), i1 = (uint32_t)min(i0_64 + t.T, (uint64_t)t.items);
    const bool active = k < a.chunks && group < groups;
    auto put = [](float *to, const float (&v)[kW][8]) {
#pragma unroll
        for (int w = 0; w < kW; ++w) put8(to + 8 * w, v[w]);
    };
    auto store = [&](uint32_t run, const float (&v)[kW][8]) {
#pragma unroll
        for (int w = 0; w < kW; ++w) sum_store<T, kVec>(t, a.C, run, group + w, v[w]);
    };
    if (active && i0 < i1) {
        const O *dy = static_cast<const O *>(a.dy);
        const DropKey key = drop_key(a.drop);
        constexpr int kBatch = 4;                             // rows that are asked for before the first is added
        OrderWalk walk(t, i0);
        uint2 next[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) next[j] = walk.next(i1);
        uint32_t run = next[0].x;
        const uint32_t head = run;
        const bool open = i0 > 0 && key_at(t, i0 - 1) == run;
        const uint32_t beyond = i1 < t.items ? key_at(t, i1) : ~0u;
        float sum[kW][8] = {};
        bool one = true;                                      // still in the first run
        auto leave = [&]() {                                  // a run that ends in the chunk
            if (one && open) put(first_sum + threadIdx.x * 8 * kW, sum);
            else if (run < t.most) store(run, sum);
        };
        for (uint32_t i = i0; i < i1; i += kBatch) {
            uint2 now[kBatch];
            Eight<O> e[kBatch][kW];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                now[j] = next[j];
                if (now[j].x < t.most)
#pragma unroll
                    for (int w = 0; w < kW; ++w) sum_load<O, kVec>(a, dy, now[j].y, group + w, e[j][w]);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) next[j] = walk.next(i1);
            auto add_row = [&](int j) {
#pragma unroll
                for (int w = 0; w < kW; ++w) {
                    float v[8];
                    floats8(e[j][w], v);
                    if (a.drop.thr) add_kept8(a.drop, key, group + w, now[j].y, v, sum[w]);
                    else
#pragma unroll
                        for (int c = 0; c < 8; ++c) sum[w][c] += v[c];
                }
            };
            bool same = run < t.most;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) same = same && now[j].x == run;
            if (same) {                                       // all of the run: no branches between the rows' generators
#pragma unroll
                for (int j = 0; j < kBatch; ++j) add_row(j);
                continue;
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (i + j >= i1) break;
                if (now[j].x != run) {
                    leave();
                    run = now[j].x;
                    one = false;
#pragma unroll
                    for (int w = 0; w < kW; ++w)
#pragma unroll
                        for (int c = 0; c < 8; ++c) sum[w][c] = 0.f;
                }
                if (run < t.most) add_row(j);
            }
        }
        const bool goes_on = i1 < t.items && beyond == run;
        if (!goes_on) leave();
        else if (one && open) put(first_sum + threadIdx.x * 8 * kW, sum);
        else put(last_sum + threadIdx.x * 8 * kW, sum);
        if (threadIdx.x == k * a.lanes) {
            first_run[k] = head;
            flags[k] = (open ? kRunOpen : 0) | (goes_on ? kRunGoesOn : 0) | (open && goes_on && one ? kRunThrough : 0);
        }
    } else if (active && threadIdx.x == k * a.lanes) {
        flags[k] = 0;
    }
    __syncthreads();
    if (a.beside_zero && blockIdx.x + 1 == gridDim.x) ptx::grid_wait();   // (what comes behind this launch comes behind that one too; the other blocks make room)
    // The first chunk's threads walk over the block's chunks: runs that begin and end in the block are finished, others leave their part.
    if (k > 0 || !active || i0 >= i1) return;
    float sum[kW][8];
    auto add = [&](const float *from) {
#pragma unroll
        for (int w = 0; w < kW; ++w) add8(sum[w], from + 8 * w);
    };
    auto clear = [&]() {
#pragma unroll
        for (int w = 0; w < kW; ++w)
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[w][c] = 0.f;
    };
    bool has = false, before = false;                         // a run is being added up; it began before the block
    float *part = t.part + (uint64_t)span * 2 * a.columns + group * 8;
    for (uint32_t c = 0; c < a.chunks; ++c) {
        const uint32_t f = flags[c], here = c * a.lanes + threadIdx.x;
        if (f & kRunOpen) {
            if (!has) {                                       // (only the first chunk's)
                clear();
                has = before = true;
            }
            add(first_sum + here * 8 * kW);
            if (!(f & kRunThrough)) {
                if (before) put(part, sum);
                else if (first_run[c] < t.most) store(first_run[c], sum);
                has = false;
            }
        }
        if ((f & kRunGoesOn) && !(f & kRunThrough)) {
            clear();
            add(last_sum + here * 8 * kW);
            has = true;
            before = false;
        }
    }
    if (has) put(part + (before ? 0 : a.columns), sum);
}
// Runs that reach over the end of a block's rows, by whoever has the span that they begin in: a warp up to kJoinShort spans, else its block.
constexpr int kJoinWarps = kTokenThreads / 32;
constexpr uint32_t kJoinShort = 8;
template <typename T, bool kVec>
__global__ void __launch_bounds__(kTokenThreads) embed_join_kernel(const SumArgs a) {
    __shared__ __align__(16) float sums[kTokenThreads][8];
    __shared__ uint32_t run_of[kJoinWarps], last_of[kJoinWarps];                // of a long run that begins in a warp's span: its key, its last span (0: none)
    if (a.beside_zero == 2) {
        __threadfence();
    } else {
        ptx::grid_launch();
        ptx::grid_wait();
    }
    const uint32_t blocks0 = (a.task[0].spans + kJoinWarps - 1) / kJoinWarps, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool second = blockIdx.x >= blocks0;
    const SumTask &t = a.task[second];
    const uint32_t first = (blockIdx.x - (second ? blocks0 : 0)) * kJoinWarps, span = first + warp, groups = a.columns / 8;
    const uint64_t rows = (uint64_t)t.T * a.chunks;
    auto part_of = [&](uint32_t c, uint32_t begin, uint32_t group) { return t.part + ((uint64_t)c * 2 + (c == begin ? 1 : 0)) * a.columns + group * 8; };
    uint32_t last = 0, run = t.most;
    const uint64_t end = (span + 1) * rows;
    if (span < t.spans && end < t.items) {
        run = key_at(t, (uint32_t)end - 1);
        const uint32_t after = key_at(t, (uint32_t)end), begin = key_at(t, (uint32_t)(span * rows)), ahead = span > 0 ? key_at(t, (uint32_t)(span * rows) - 1) : ~run;
        if (run < t.most && after == run && !(begin == run && ahead == run)) {
            // its last span: the last one that begins with it; 32 candidates at a time, the distance between them 32 times as large whenever all are
            last = span + 1;
            uint32_t step = 1;
            while (true) {
                const uint64_t c = (uint64_t)last + (uint64_t)(lane + 1) * step;
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, c < t.spans && key_at(t, (uint32_t)(c * rows)) == run));   // (sorted: the first n of them)
                last += n * step;
                if (n == 32) step *= 32;
                else if (step == 1) break;
                else step /= 32;
            }
        }
    }
    const bool is_long = last > 0 && last - span + 1 > kJoinShort;
    if (lane == 0) { run_of[warp] = run; last_of[warp] = is_long ? last : 0; }
    if (last > 0 && !is_long)
        for (uint32_t group = lane; group < groups; group += 32) {
            float s[8] = {};
            float4 p[kJoinShort][2];
#pragma unroll
            for (uint32_t i = 0; i < kJoinShort; ++i) {
                const float4 *from = reinterpret_cast<const float4 *>(part_of(min(span + i, last), span, group));
                p[i][0] = from[0]; p[i][1] = from[1];
            }
#pragma unroll
            for (uint32_t i = 0; i < kJoinShort; ++i)
                if (span + i <= last) {
                    s[0] += p[i][0].x; s[1] += p[i][0].y; s[2] += p[i][0].z; s[3] += p[i][0].w;
                    s[4] += p[i][1].x; s[5] += p[i][1].y; s[6] += p[i][1].z; s[7] += p[i][1].w;
                }
            sum_store<T, kVec>(t, a.C, run, group, s);
        }
    __syncthreads();
    // groups of columns that the block has side by side (a power of two, 16 to 128), and spans
    uint32_t side = 16;
    while (side < 128 && side < groups) side *= 2;
    const uint32_t column = threadIdx.x & (side - 1), slice = threadIdx.x / side, slices = kTokenThreads / side;
    for (uint32_t k = 0; k < kJoinWarps; ++k) {
        if (last_of[k] == 0) continue;
        for (uint32_t g0 = 0; g0 < groups; g0 += side) {
            const uint32_t group = g0 + column;
            float s[8] = {};
            if (group < groups)
#pragma unroll 8
                for (uint32_t c = first + k + slice; c <= last_of[k]; c += slices) add8(s, part_of(c, first + k, group));
            put8(sums[threadIdx.x], s);
            __syncthreads();
            if (slice == 0 && group < groups) {
                for (uint32_t r = 1; r < slices; ++r) add8(s, sums[r * side + column]);
                sum_store<T, kVec>(t, a.C, run_of[k], group, s);
            }
            __syncthreads();
        }
    }
    if (a.beside_zero == 2 && blockIdx.x + 1 == gridDim.x) ptx::grid_wait();
}

}  // namespace flare
