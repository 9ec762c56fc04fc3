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

// Generator and threshold; thr = 0: nothing is dropped.
struct DropArgs {
    uint32_t thr;
    float keep;
    uint64_t seed, offset;
    const int64_t *step;                                      // device, or null: added to offset
};
struct DropKey { uint32_t k0, k1, c2, c3; };
__device__ __forceinline__ DropKey drop_key(const DropArgs &d) {
    const uint64_t at = d.offset + (d.thr != 0 && d.step != nullptr ? (uint64_t)*d.step : 0ull);
    return DropKey{(uint32_t)d.seed, (uint32_t)(d.seed >> 32), (uint32_t)at, (uint32_t)(at >> 32)};
}
__device__ __forceinline__ uint4 philox(const DropKey &k, uint32_t group, uint32_t row) {
    uint32_t c0 = group, c1 = row, c2 = k.c2, c3 = k.c3, k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Eight columns' values through dropout: what is dropped is 0 whatever it was.
__device__ __forceinline__ void drop8(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row, float (&v)[8]) {
    const uint4 u = philox(k, group, row);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (w[i] & 0xffffu) >= d.thr ? v[2 * i] * d.keep : 0.f;
        v[2 * i + 1] = (w[i] >> 16) >= d.thr ? v[2 * i + 1] * d.keep : 0.f;
    }
}
// The same as eight bits.
__device__ __forceinline__ uint32_t keep8(const DropArgs &d, const DropKey &k, uint32_t group, uint32_t row) {
    const uint4 u = philox(k, group, row);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= ((w[i] & 0xffffu) >= d.thr ? 1u : 0u) << (2 * i);
        bits |= ((w[i] >> 16) >= d.thr ? 1u : 0u) << (2 * i + 1);
    }
    return bits;
}

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
    __device__ __forceinline__ void next() {
        row += drow; group += dgroup;
        if (group >= groups) { group -= groups; ++row; }
    }
};

// ---------------------------------------------------------------- dropout
struct DropoutArgs {
    const void *x, *residual;                                 // residual: null if there is none
    void *y;
    long ld_x, ld_r, ld_y;
    uint32_t rows, C;
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
                    load8(x + (long)w.row * a.ld_x + w.group * 8, e[k]);
                    if (res) load8(res + (long)w.row * a.ld_r + w.group * 8, f[k]);
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
                store8(y + (long)row[k] * a.ld_y + group[k] * 8, v);
            }
        }
    } else {
        const uint32_t lane = threadIdx.x & 31, warps = kTokenThreads / 32;
        GroupWalk w((uint64_t)blockIdx.x * warps + (threadIdx.x >> 5), (uint64_t)gridDim.x * warps, (a.C + 255) / 256);
        for (; w.row < a.rows; w.next()) {
            const uint32_t c0 = w.group * 256 + lane;
            const X *px = x + (long)w.row * a.ld_x + c0;
            const R *pr = res ? res + (long)w.row * a.ld_r + c0 : nullptr;
            R *py = y + (long)w.row * a.ld_y + c0;
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

// ---------------------------------------------------------------- embedding, forward
struct EmbedArgs {
    const void *tokens, *table, *positions;                   // positions: null if there are none
    void *y;
    long ld_t, ld_y;
    uint32_t rows, C, L;                                      // L: positions, row n takes n mod L
    int64_t vocab;
    float scale;
    DropArgs drop;
    int wide;                                                 // tokens are 64 bits
};
__device__ __forceinline__ int64_t token_at(const void *tokens, int wide, uint32_t n) {
    return wide ? static_cast<const int64_t *>(tokens)[n] : (int64_t) static_cast<const int32_t *>(tokens)[n];
}
// T: type of the tables, O: of the rows.
template <typename T, typename O, bool kVec>
__global__ void __launch_bounds__(kTokenThreads) embed_kernel(const EmbedArgs a) {
    ptx::grid_launch();
    ptx::grid_wait();
    const T *table = static_cast<const T *>(a.table), *pos = static_cast<const T *>(a.positions);
    O *y = static_cast<O *>(a.y);
    const DropKey key = drop_key(a.drop);
    if constexpr (kVec) {
        constexpr int kBatch = 4;
        GroupWalk w((uint64_t)blockIdx.x * kTokenThreads + threadIdx.x, (uint64_t)gridDim.x * kTokenThreads, a.C / 8);
        while (w.row < a.rows) {
            uint32_t row[kBatch], group[kBatch];
            int64_t t[kBatch];
            Eight<T> e[kBatch], f[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                row[k] = w.row; group[k] = w.group;
                t[k] = -1;
                if (w.row < a.rows) t[k] = token_at(a.tokens, a.wide, w.row);
                w.next();
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (t[k] >= 0 && t[k] < a.vocab) load8(table + t[k] * a.ld_t + group[k] * 8, e[k]);
                if (pos && row[k] < a.rows) load8(pos + (long)(row[k] % a.L) * a.C + group[k] * 8, f[k]);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (row[k] >= a.rows) break;
                float v[8] = {};
                if (t[k] >= 0 && t[k] < a.vocab) {
                    floats8(e[k], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= a.scale;
                }
                if (pos) {
                    float r[8];
                    floats8(f[k], r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += r[i];
                }
                if (a.drop.thr) drop8(a.drop, key, group[k], row[k], v);
                store8(y + (long)row[k] * a.ld_y + group[k] * 8, v);
            }
        }
    } else {
        const uint32_t lane = threadIdx.x & 31, warps = kTokenThreads / 32;
        GroupWalk w((uint64_t)blockIdx.x * warps + (threadIdx.x >> 5), (uint64_t)gridDim.x * warps, (a.C + 255) / 256);
        for (; w.row < a.rows; w.next()) {
            const uint32_t c0 = w.group * 256 + lane;
            const int64_t t = token_at(a.tokens, a.wide, w.row);
            const bool there = t >= 0 && t < a.vocab;
            const T *pe = table + (there ? t * a.ld_t + c0 : 0), *pp = pos ? pos + (long)(w.row % a.L) * a.C + c0 : nullptr;
            O *py = y + (long)w.row * a.ld_y + c0;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool in = c0 + 32 * k < a.C;
                v[k] = there && in ? to_f32(pe[32 * k]) * a.scale : 0.f;
                if (pp && in) v[k] += to_f32(pp[32 * k]);
            }
            const uint32_t bits = a.drop.thr ? keep8(a.drop, key, w.group * 32 + lane, w.row) : 0xffu;
            const float keep = a.drop.thr ? a.drop.keep : 1.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t b = __shfl_sync(0xffffffffu, bits, 4 * k + (lane >> 3));
                const float d = b >> (lane & 7) & 1 ? v[k] * keep : 0.f;
                if (c0 + 32 * k < a.C) from_f32(py[32 * k], d);
            }
        }
    }
}

// ---------------------------------------------------------------- embedding, backward
//
// Rows that met the same token are added up in the order of the rows, whatever else the GPU does: the tokens are sorted (stably), the sorted rows are cut
// into chunks of the same length, and a thread adds up eight columns of a chunk's rows.  A token all of whose rows lie in one chunk is finished there;
// one that reaches over a chunk's end leaves float32 sums, which a second kernel adds up in the order of the chunks.  So a token that every third row has
// takes no longer than rare ones, and no sum depends on the order in which blocks run.
//
// Positions are the same with an order that need not be sorted: row i of it is row (i mod B) L + i / B of the batch, its "token" i / B.
//
// The sort: one cluster of blocks (up to 16 of 1024 threads), each a stretch of the tokens, each of its warps a stretch of that.  A pass over a digit of up to
// ten bits: every warp counts its stretch (lanes with the same digit find one another by match.any, so a warp's counts need no atomics), the counts before it
// are added up over the warps in shared memory and over the blocks through distributed shared memory, and every warp puts its tokens where those say.  One
// launch, two barriers of the cluster a pass, where kernels of a count, a scan and a scatter each would be three launches a pass; meanwhile the other
// clusters of the same launch set the gradient to zero, which a large vocabulary needs longer for than the sort takes.
constexpr int kSortThreads = 1024, kSortBits = 10, kSortBatch = 8;
struct SortArgs {
    const void *tokens;
    int wide;
    uint32_t rows;
    int64_t vocab;
    int passes, bits;                                         // digits of the key (a token in range, or vocab for one that is not)
    uint32_t *key[2], *index[2];                              // the last pass writes to [passes & 1 ? 0 : 1]; see sorted_in
    uint4 *zero;                                              // what the other clusters set to zero, as 16-byte words
    uint64_t zeros;
    uint8_t *tail;                                            // and bytes beyond those, and before
    uint8_t *head;
    uint32_t tails, heads;
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

__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const SortArgs a) {
    extern __shared__ uint32_t counts[];                      // [32 warps][bins], then [bins] of the block, [32] of a scan
    ptx::grid_launch();
    ptx::grid_wait();
    const uint32_t blocks = ptx::cluster_size(), rank = ptx::cluster_rank();
    if (blockIdx.x >= blocks) {
        const uint64_t n = (uint64_t)(gridDim.x - blocks) * kSortThreads, me = (uint64_t)(blockIdx.x - blocks) * kSortThreads + threadIdx.x;
        for (uint64_t i = me; i < a.zeros; i += n) a.zero[i] = make_uint4(0, 0, 0, 0);
        if (me < a.heads) a.head[me] = 0;
        if (me < a.tails) a.tail[me] = 0;
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // stretches: of a block, of a warp (whole groups of 32)
    const uint32_t per_warp = ((a.rows + blocks * 32 - 1) / (blocks * 32) + 31) / 32 * 32;
    const uint64_t first64 = (uint64_t)(rank * 32 + warp) * per_warp;
    const uint32_t first = (uint32_t)min(first64, (uint64_t)a.rows), last = (uint32_t)min(first64 + per_warp, (uint64_t)a.rows);
    const uint32_t bins = 1u << a.bits;
    uint32_t *mine = counts + warp * bins, *block = counts + 32 * bins, *scan = block + bins;
    for (int pass = 0; pass < a.passes; ++pass) {
        const uint32_t shift = pass * a.bits;
        const uint32_t *key_in = a.key[(pass & 1) ^ 1], *index_in = a.index[(pass & 1) ^ 1];
        uint32_t *key_out = a.key[pass & 1], *index_out = a.index[pass & 1];
        auto key_of = [&](uint32_t i) -> uint32_t {
            if (pass > 0) return __ldcg(key_in + i);
            const int64_t t = token_at(a.tokens, a.wide, i);
            return t >= 0 && t < a.vocab ? (uint32_t)t : (uint32_t)a.vocab;
        };
        for (uint32_t i = threadIdx.x; i < 32 * bins; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        // (kSortBatch groups of 32 are asked for before the first is looked at)
        for (uint32_t i0 = first; i0 < last; i0 += 32 * kSortBatch) {
            uint32_t digit[kSortBatch];
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) digit[j] = i0 + 32 * j + lane < last ? key_of(i0 + 32 * j + lane) >> shift & (bins - 1) : ~0u;
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                if (i0 + 32 * j >= last) break;
                const uint32_t same = __match_any_sync(0xffffffffu, digit[j]);
                if (digit[j] != ~0u && (same & ((1u << lane) - 1)) == 0) mine[digit[j]] += __popc(same);
                __syncwarp();
            }
        }
        __syncthreads();
        // before each warp within the block
        const uint32_t d = threadIdx.x;
        uint32_t total = 0;
        if (d < bins) {
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
            for (uint32_t r = 0; r < blocks; ++r) {
                const uint32_t c = ptx::lds_cluster(ptx::in_block(ptx::smem_u32(block + d), r));
                if (r < rank) before += c;
                all += c;
            }
        }
        // before each digit: a scan over the block's threads
        uint32_t sum = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= (uint32_t)o) sum += up;
        }
        if (lane == 31) scan[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            uint32_t s = scan[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t up = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= (uint32_t)o) s += up;
            }
            scan[lane] = s;
        }
        __syncthreads();
        if (d < bins) {
            const uint32_t base = before + sum - all + (warp > 0 ? scan[warp - 1] : 0);
            for (uint32_t w = 0; w < 32; ++w) counts[w * bins + d] += base;
        }
        __syncthreads();
        for (uint32_t i0 = first; i0 < last; i0 += 32 * kSortBatch) {
            uint32_t key[kSortBatch], index[kSortBatch];
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                const uint32_t i = i0 + 32 * j + lane;
                key[j] = i < last ? key_of(i) : 0u;
                index[j] = i < last && pass > 0 ? __ldcg(index_in + i) : i;
            }
#pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                if (i0 + 32 * j >= last) break;
                const bool in = i0 + 32 * j + lane < last;
                const uint32_t digit = in ? key[j] >> shift & (bins - 1) : ~0u;
                const uint32_t same = __match_any_sync(0xffffffffu, digit), lower = same & ((1u << lane) - 1);
                uint32_t at = 0;
                if (in) at = mine[digit] + __popc(lower);
                __syncwarp();
                if (in) {
                    if (lower == 0) mine[digit] += __popc(same);
                    key_out[at] = key[j];
                    index_out[at] = index[j];
                }
                __syncwarp();
            }
        }
        // (what was put into memory is seen by all blocks; nobody's counts are read any more)
        ptx::cluster_meet();
    }
}

// Sums over runs of equal keys.  Two tasks in one launch: tokens, and positions.
struct SumTask {
    const uint32_t *key, *index;                              // sorted; null: positions
    uint32_t items, batch, L;                                 // items of the order; positions: batch items, rows of an item
    uint32_t most;                                            // keys from here on are none
    void *out;
    long ld_out;
    float scale;
    int add;                                                  // to what is there
    float *part;                                              // [chunks][2][columns]: of the run a chunk begins with, of the one it ends with
    uint32_t chunks, blocks;
};
struct SumArgs {
    SumTask task[2];
    const void *dy;
    long ld_dy;
    uint32_t C, columns, T;                                   // columns: C up to whole groups of eight; T: rows of a chunk
    DropArgs drop;
};
struct SumOrder {
    const uint32_t *key, *index;
    uint32_t batch, L;
    __device__ __forceinline__ explicit SumOrder(const SumTask &t) : key(t.key), index(t.index), batch(t.batch), L(t.L) {}
    __device__ __forceinline__ uint32_t key_at(uint32_t i) const { return key ? key[i] : i / batch; }
    __device__ __forceinline__ uint32_t row_at(uint32_t i) const { return key ? index[i] : i % batch * L + i / batch; }
};
// kVec: dy's rows on 16-byte boundaries and C a multiple of 8; out8: out's too.
template <typename O, typename T, bool kVec>
__device__ __forceinline__ void sum_load(const SumArgs &a, const O *dy, uint32_t row, uint32_t group, Eight<O> &e) {
    const O *p = dy + (long)row * a.ld_dy + group * 8;
    if constexpr (kVec) load8(p, e);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (group * 8 + i < a.C) reinterpret_cast<O *>(e.q)[i] = p[i];
            else from_f32(reinterpret_cast<O *>(e.q)[i], 0.f);
    }
}
template <typename T, bool kVec>
__device__ __forceinline__ void sum_store(const SumTask &t, uint32_t C, uint32_t key, uint32_t group, float (&v)[8]) {
    T *p = static_cast<T *>(t.out) + (long)key * t.ld_out + group * 8;
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
template <typename O, typename T, bool kVec>
__global__ void __launch_bounds__(kTokenThreads) embed_sum_kernel(const SumArgs a) {
    ptx::grid_launch();
    ptx::grid_wait();
    const bool second = blockIdx.x >= a.task[0].blocks;
    const SumTask &t = a.task[second];
    const uint32_t groups = a.columns / 8;
    const uint64_t at = (uint64_t)(blockIdx.x - (second ? a.task[0].blocks : 0)) * kTokenThreads + threadIdx.x;
    const uint64_t chunk64 = at / groups;
    if (chunk64 >= t.chunks) return;
    const uint32_t chunk = (uint32_t)chunk64, group = (uint32_t)(at - chunk64 * groups), i0 = chunk * a.T, i1 = (uint32_t)min((uint64_t)i0 + a.T, (uint64_t)t.items);
    const SumOrder order(t);
    const O *dy = static_cast<const O *>(a.dy);
    const DropKey key = drop_key(a.drop);
    uint32_t run = order.key_at(i0);
    bool open = i0 > 0 && order.key_at(i0 - 1) == run;        // the run began before the chunk
    float sum[8] = {};
    auto leave = [&](bool goes_on) {
        if (run >= t.most) return;
        if (open || goes_on) {
            float4 *p = reinterpret_cast<float4 *>(t.part + ((uint64_t)chunk * 2 + (open ? 0 : 1)) * a.columns + group * 8);
            p[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            p[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        } else {
            sum_store<T, kVec>(t, a.C, run, group, sum);
        }
    };
    constexpr int kBatch = 4;
    for (uint32_t i = i0; i < i1; i += kBatch) {
        uint32_t k[kBatch], row[kBatch];
        Eight<O> e[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            k[j] = i + j < i1 ? order.key_at(i + j) : ~0u;
            row[j] = i + j < i1 ? order.row_at(i + j) : 0u;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (k[j] < t.most) sum_load<O, T, kVec>(a, dy, row[j], group, e[j]);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (i + j >= i1) break;
            if (k[j] != run) {
                leave(false);
                run = k[j];
                open = false;
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] = 0.f;
            }
            if (k[j] >= t.most) continue;
            float v[8];
            floats8(e[j], v);
            if (a.drop.thr) drop8(a.drop, key, group, row[j], v);
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] += v[c];
        }
    }
    leave(i1 < t.items && order.key_at(i1) == run);
}
// Runs that reach over a chunk's end: by the block of the chunk that they begin in, kJoinRows chunks at a time.
constexpr int kJoinColumns = 16, kJoinRows = kTokenThreads / kJoinColumns;      // groups of eight columns, chunks, that a block has side by side
template <typename T, bool kVec>
__global__ void __launch_bounds__(kTokenThreads) embed_join_kernel(const SumArgs a) {
    __shared__ float sums[kJoinRows][kJoinColumns * 8];
    ptx::grid_launch();
    ptx::grid_wait();
    const bool second = blockIdx.x >= a.task[0].chunks;
    const SumTask &t = a.task[second];
    const uint32_t chunk = blockIdx.x - (second ? a.task[0].chunks : 0);
    const SumOrder order(t);
    const uint64_t end = (uint64_t)(chunk + 1) * a.T;
    if (end >= t.items) return;
    const uint32_t run = order.key_at((uint32_t)end - 1);
    if (run >= t.most || order.key_at((uint32_t)end) != run) return;                   // no run reaches over the end
    if (order.key_at(chunk * a.T) == run && chunk > 0 && order.key_at(chunk * a.T - 1) == run) return;   // it began before this chunk
    // the run's last chunk: the last one that begins with it
    uint32_t lo = chunk + 1, hi = t.chunks - 1;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        if (order.key_at(mid * a.T) == run) lo = mid;
        else hi = mid - 1;
    }
    const uint32_t lane = threadIdx.x % kJoinColumns, slice = threadIdx.x / kJoinColumns, groups = a.columns / 8;
    for (uint32_t g0 = 0; g0 < groups; g0 += kJoinColumns) {
        const uint32_t group = g0 + lane;
        float sum[8] = {};
        if (group < groups)
#pragma unroll 4
            for (uint32_t c = chunk + slice; c <= lo; c += kJoinRows) {
                const float4 *p = reinterpret_cast<const float4 *>(t.part + ((uint64_t)c * 2 + (c == chunk ? 1 : 0)) * a.columns + group * 8);
                const float4 x = p[0], y = p[1];
                sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
                sum[4] += y.x; sum[5] += y.y; sum[6] += y.z; sum[7] += y.w;
            }
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[slice][lane * 8 + i] = sum[i];
        __syncthreads();
        if (slice == 0 && group < groups) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float s = 0.f;
#pragma unroll
                for (int r = 0; r < kJoinRows; ++r) s += sums[r][lane * 8 + i];
                sum[i] = s;
            }
            sum_store<T, kVec>(t, a.C, run, group, sum);
        }
        __syncthreads();
    }
}

}  // namespace flare
