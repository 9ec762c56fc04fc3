// Embedding lookup, its gradient and dropout: argument checks, workspace, launches.
#include "flare_host.h"
#include "flare_tokens.cuh"

namespace flare {
namespace {

size_t size_of(int dtype) { return dtype == FLARE_DTYPE_F32 ? 4 : 2; }
bool a_type(int t) { return t == FLARE_DTYPE_F32 || t == FLARE_DTYPE_BF16 || t == FLARE_DTYPE_F16; }
bool natural(const void *p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }
// Rows that can be moved 16 bytes at a time.
bool rows16(const void *p, long ld, size_t size) { return aligned16(p) && ld * size % 16 == 0; }

int need_device() {
    const DeviceView di = device_info();
    if (di.checked == -2) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "no CUDA device");
        return FLARE_ERR_CUDA;
    }
    return di.checked == 1 ? FLARE_OK : FLARE_ERR_ARCH;
}

int check_drop(const flare_drop_t *d) {
    if (d == nullptr) return FLARE_OK;
    return d->p >= 0.f && d->p <= 1.f && natural(d->step, 8) ? FLARE_OK : FLARE_ERR_INVALID_ARG;
}
DropArgs drop_args(const flare_drop_t *d) {
    DropArgs a{};
    a.keep = 1.f;
    if (d == nullptr) return a;
    a.thr = (uint32_t)std::lrint((double)d->p * 65536.0);
    a.keep = a.thr < 65536 ? (float)(65536.0 / (65536 - a.thr)) : 0.f;
    for (uint32_t r = 0; r < 10; ++r) {
        a.k0[r] = (uint32_t)d->seed + r * 0x9E3779B9u;
        a.k1[r] = (uint32_t)(d->seed >> 32) + r * 0xBB67AE85u;
    }
    a.offset = d->offset; a.step = d->step;
    return a;
}
// Blocks of a kernel that walks over `items`: a thread an item, or sixteen blocks an SM (up to four of them at a time).
unsigned walk_blocks(uint64_t items, int per_block) { return (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((items + per_block - 1) / per_block, 16ull * device_info().sms)); }

int check_dropout(const flare_dropout_desc_t *d) {
    if (d == nullptr || d->rows < 0 || d->width <= 0) return FLARE_ERR_INVALID_ARG;
    for (int64_t s : {d->stride_x, d->stride_residual, d->stride_y})
        if (s != 0 && s < d->width) return FLARE_ERR_INVALID_ARG;
        else if (s > INT32_MAX) return FLARE_ERR_UNSUPPORTED;
    if (!a_type(d->dtype) || (d->residual_dtype != d->dtype && d->residual_dtype != FLARE_DTYPE_F32)) return FLARE_ERR_UNSUPPORTED;
    return d->rows > ((int64_t)1 << 31) - 1 ? FLARE_ERR_UNSUPPORTED : FLARE_OK;
}

template <typename X, typename R>
int launch_dropout(const DropoutArgs &a, bool vec, cudaStream_t st) {
    // one long row: some 4096 elements a block, of at least eight rows, whose bits fit shared memory
    const bool flat = !vec && a.drop.thr && aligned16(a.x) && aligned16(a.residual) && aligned16(a.y) && a.ld_x == a.C && a.ld_y == a.C && (!a.residual || a.ld_r == a.C);
    if (flat && a.C >= 8 && a.C <= 32768) {
        DropoutFlat f{a, std::max(8u, 4096u / a.C / 8 * 8)};
        FLARE_CUDA(launch_after(dropout_flat_kernel<X, R>, (a.rows + f.tile_rows - 1) / f.tile_rows, kTokenThreads, ((size_t)f.tile_rows * a.C + 31) / 32 * 4, st, f));
        return FLARE_OK;
    }
    if (vec) FLARE_CUDA(launch_after(dropout_kernel<X, R, true>, walk_blocks((uint64_t)a.rows * (a.C / 8), kTokenThreads), kTokenThreads, 0, st, a));
    else FLARE_CUDA(launch_after(dropout_kernel<X, R, false>, walk_blocks((uint64_t)a.rows * ((a.C + 255) / 256), kTokenThreads / 32), kTokenThreads, 0, st, a));
    return FLARE_OK;
}
// The two types of an operator: equal, or one of them float32.
#define FLARE_TWO_TYPES(a, b, call)                                                                                         \
    ((a) == FLARE_DTYPE_F32    ? ((b) == FLARE_DTYPE_F32 ? call<float, float> : (b) == FLARE_DTYPE_BF16 ? call<float, __nv_bfloat16> : call<float, __half>) \
     : (a) == FLARE_DTYPE_BF16 ? ((b) == FLARE_DTYPE_F32 ? call<__nv_bfloat16, float> : call<__nv_bfloat16, __nv_bfloat16>) \
                               : ((b) == FLARE_DTYPE_F32 ? call<__half, float> : call<__half, __half>))

int check_embed(const flare_embed_desc_t *d) {
    if (d == nullptr || d->rows < 0 || d->width <= 0 || d->vocab <= 0 || d->positions < 0 || !std::isfinite(d->scale)) return FLARE_ERR_INVALID_ARG;
    if (d->positions > 0 && d->rows % d->positions != 0) return FLARE_ERR_INVALID_ARG;
    if (d->token_bits != 32 && d->token_bits != 64) return FLARE_ERR_INVALID_ARG;
    for (int64_t s : {d->stride_table, d->stride_out})
        if (s != 0 && s < d->width) return FLARE_ERR_INVALID_ARG;
        else if (s > INT32_MAX) return FLARE_ERR_UNSUPPORTED;
    if (!a_type(d->dtype) || !a_type(d->out_dtype)) return FLARE_ERR_UNSUPPORTED;
    if (d->dtype != d->out_dtype && d->dtype != FLARE_DTYPE_F32 && d->out_dtype != FLARE_DTYPE_F32) return FLARE_ERR_UNSUPPORTED;
    return d->rows > ((int64_t)1 << 31) - 1 || d->width > (1 << 20) ? FLARE_ERR_UNSUPPORTED : FLARE_OK;
}

template <typename T, typename O>
int launch_embed(const EmbedArgs &a, bool vec, cudaStream_t st) {
    // (two groups a thread where there are enough of them to keep every SM busy with half as many threads: 4096 rows of 512 take 6.2 us, one a thread 7.3; 131072 of 128 18.9 and 20.2; half as many as that no
    // difference)
    const uint64_t groups = (uint64_t)a.rows * (a.C / 8);
    if (vec && a.C % 16 == 0 && groups >= 1024ull * device_info().sms)
        FLARE_CUDA(launch_after(embed_kernel<T, O, 2>, walk_blocks(groups / 2, kTokenThreads), kTokenThreads, 0, st, a));
    else if (vec) FLARE_CUDA(launch_after(embed_kernel<T, O, 1>, walk_blocks(groups, kTokenThreads), kTokenThreads, 0, st, a));
    else FLARE_CUDA(launch_after(embed_kernel<T, O, 0>, walk_blocks((uint64_t)a.rows * ((a.C + 255) / 256), kTokenThreads / 32), kTokenThreads, 0, st, a));
    return FLARE_OK;
}

// Two groups a thread where that leaves a row 32 threads, and an SM some 256; 16-bit gradients (float32 ones would not fit the registers).
bool sum_in_twos(const flare_embed_desc_t *d, int sms) {
    return d->width % 16 == 0 && d->width >= 512 && d->out_dtype != FLARE_DTYPE_F32 && d->rows * (d->width / 16) >= 8L * 256 * sms;
}
// How the sums' blocks lie over the columns and along the order.
struct SumShape { uint32_t threads, lanes, tiles, chunks; };
SumShape sum_shape(const flare_embed_desc_t *d, bool twos) {
    const uint32_t units = twos ? (uint32_t)d->width / 16 : ((uint32_t)d->width + 7) / 8, threads = units <= 16 ? 128 : kSumThreads;
    const uint32_t tiles = (units + threads - 1) / threads, lanes = (units + tiles - 1) / tiles;
    return SumShape{threads, lanes, tiles, threads / lanes};
}
// Rows of a chunk of the backward's sums: such that an SM has some 1024 groups of columns, 16 to 64.  Positions: whole runs (one row of every batch item) where they are not longer than that, so
// that none reaches over a chunk's end.
int chunk_rows(const flare_embed_desc_t *d, int sms) {
    const long want = d->rows * ((d->width + 7) / 8) / (1024L * sms), T = std::min(64L, std::max(16L, want / 4 * 4));
    if (!sum_in_twos(d, sms)) return (int)T;
    // Longer, where the blocks of wide rows, two an SM, would be a third of a round or less more than whole rounds: 65536 rows of 512 over 256 words take 51 us in chunks of 24 rows (342 blocks for 296 places), 44.6 of
    // 28.  (Narrow ones are more and smaller: 131072 rows of 128 over 32000 words took 66.5 instead of 63.7, over 256 words 38.9 instead of 40.2.)
    const SumShape s = sum_shape(d, true);
    const long blocks = (d->rows * s.tiles + T * s.chunks - 1) / (T * s.chunks), places = 2L * sms, rounds = blocks / places;
    if (rounds < 1 || blocks - rounds * places > places / 3) return (int)T;
    const long fit = s.chunks * places * rounds;
    return (int)std::min(64L, ((d->rows * s.tiles + fit - 1) / fit + 3) / 4 * 4);
}
int chunk_rows_of_positions(const flare_embed_desc_t *d, int sms) {
    const long T = chunk_rows(d, sms), batch = d->positions > 0 ? d->rows / d->positions : 1;
    return (int)(batch > 64 || batch < 1 ? T : std::max(1L, T / batch) * batch);
}
struct EmbedLayout { size_t pairs[2], part[2], total; long spans[2]; };
EmbedLayout embed_layout(const flare_embed_desc_t *d, int sms, bool twos) {
    EmbedLayout w{};
    size_t off = kHeaderBytes;
    for (size_t &p : w.pairs) { p = off; off += align_up(sizeof(uint2) * (size_t)d->rows); }
    const int T[2] = {chunk_rows(d, sms), chunk_rows_of_positions(d, sms)};
    for (int i = 0; i < 2; ++i) {
        const long rows = (long)T[i] * sum_shape(d, twos).chunks;
        w.spans[i] = (d->rows + rows - 1) / rows;
        w.part[i] = off;
        if (i == 0 || d->positions > 0) off += align_up(sizeof(float) * 2 * (size_t)w.spans[i] * ((d->width + 7) / 8 * 8));
    }
    w.total = off;
    return w;
}

// Blocks of the cluster that sorts: sixteen where the device places them, else eight; asked for once per device, 0 = not yet.
int sort_cluster(size_t smem) {
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return 8;
    }
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 16; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(16); cfg.blockDim = kSortThreads; cfg.dynamicSmemBytes = smem;
        cfg.attrs = &attr; cfg.numAttrs = 1;
        int most = 0;
        n = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&most, embed_sort_kernel, &cfg) == cudaSuccess && most >= 1 ? 16 : 8;
        cudaGetLastError();
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}
constexpr size_t kSortSmem = sizeof(uint32_t) * ((34u << kSortBits) + 64) + sizeof(uint2) * kSortStaged;

int launch_sort(SortArgs s, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    if (int rc = ensure_big_smem(embed_sort_kernel, opt_in, (int)kSortSmem)) return rc;
    const int n = sort_cluster(kSortSmem);
    const uint64_t warps = 32ull * n, per_warp = ((s.rows + warps - 1) / warps + 31) / 32 * 32;   // (as the kernel has it)
    s.staged = 32 * per_warp <= kSortStaged;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = n; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)n);
    cfg.blockDim = kSortThreads; cfg.dynamicSmemBytes = sizeof(uint32_t) * ((34u << s.bits) + 64) + (s.staged ? sizeof(uint2) * kSortStaged : 0); cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, embed_sort_kernel, s));
    return FLARE_OK;
}

template <typename T>
int launch_zero(ZeroArgs z, uint32_t first, uint32_t last, cudaStream_t st) {
    z.first = first; z.last = last;
    const unsigned blocks = std::max(1u, std::min((last - first + kZeroThreads / 32 - 1) / (kZeroThreads / 32), 8u * device_info().sms));
    FLARE_CUDA(launch_after(sizeof(T) == 4 ? embed_zero_kernel<uint32_t> : embed_zero_kernel<uint16_t>, blocks, kZeroThreads, 0, st, z));
    return FLARE_OK;
}
// dy's type first
template <typename O, typename T>
int launch_sum(const SumArgs &a, int width, cudaStream_t st) {
    const unsigned blocks = (a.task[0].spans + a.task[1].spans) * a.tiles;
    if (width == 0) FLARE_CUDA(launch_after(embed_sum_kernel<O, T, 0>, blocks, a.threads, sum_smem(a.threads, 1), st, a));
    else if (width == 1) FLARE_CUDA(launch_after(embed_sum_kernel<O, T, 1>, blocks, a.threads, sum_smem(a.threads, 1), st, a));
    else if constexpr (sizeof(O) == 2) FLARE_CUDA(launch_after(embed_sum_kernel<O, T, 2>, blocks, a.threads, sum_smem(a.threads, 2), st, a));
    return FLARE_OK;
}
template <typename O, typename T>
int launch_sums(const SumArgs &a, const ZeroArgs &z, int width, bool whole_positions, cudaStream_t st) {
    auto joins = [](const SumTask &t) { return (t.spans + kJoinWarps - 1) / kJoinWarps; };
    const unsigned joined = joins(a.task[0]) + (whole_positions ? 0 : joins(a.task[1]));
    // positions first, beside the sort, which they need not wait for (where there is one: of a few SMs); what comes behind them comes behind it
    SumArgs positions = a;
    positions.task[0].spans = 0;
    positions.beside_zero = a.task[0].spans ? 1 : 0;
    if (positions.task[1].spans)
        if (int rc = launch_sum<O, T>(positions, width, st)) return rc;
    const uint32_t half = a.beside_zero == 2 ? z.last / 2 : z.last;
    if (a.beside_zero)
        if (int rc = launch_zero<T>(z, 0, half, st)) return rc;
    SumArgs tokens = a;
    tokens.task[1].spans = 0;
    if (tokens.task[0].spans)
        if (int rc = launch_sum<O, T>(tokens, width, st)) return rc;
    if (a.beside_zero == 2)
        if (int rc = launch_zero<T>(z, half, z.last, st)) return rc;
    if (joined && width) FLARE_CUDA(launch_after(embed_join_kernel<T, true>, joined, kTokenThreads, 0, st, a));
    else if (joined) FLARE_CUDA(launch_after(embed_join_kernel<T, false>, joined, kTokenThreads, 0, st, a));
    return FLARE_OK;
}

}  // namespace
}  // namespace flare

using namespace flare;

extern "C" {

int flare_dropout_forward(const flare_dropout_desc_t *desc, const flare_drop_t *drop, const void *x, const void *residual, void *y, flare_stream_t stream) {
    if (int rc = check_dropout(desc)) return rc;
    if (drop == nullptr) return FLARE_ERR_INVALID_ARG;
    if (int rc = check_drop(drop)) return rc;
    const size_t t = size_of(desc->dtype), r = size_of(desc->residual_dtype);
    if ((desc->rows > 0 && (!x || !y)) || !natural(x, t) || !natural(residual, r) || !natural(y, r)) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    if (desc->rows == 0) return FLARE_OK;
    DropoutArgs a{};
    auto ld = [&](int64_t s) { return (uint32_t)(s ? s : desc->width); };
    a.x = x; a.residual = residual; a.y = y;
    a.ld_x = ld(desc->stride_x); a.ld_r = ld(desc->stride_residual); a.ld_y = ld(desc->stride_y);
    a.rows = (uint32_t)desc->rows; a.C = (uint32_t)desc->width; a.drop = drop_args(drop);
    const bool vec = desc->width % 8 == 0 && rows16(x, a.ld_x, t) && rows16(y, a.ld_y, r) && (!residual || rows16(residual, a.ld_r, r));
    return FLARE_TWO_TYPES(desc->dtype, desc->residual_dtype, launch_dropout)(a, vec, reinterpret_cast<cudaStream_t>(stream));
}

int flare_dropout_backward(const flare_dropout_desc_t *desc, const flare_drop_t *drop, const void *dy, void *dx, flare_stream_t stream) {
    if (int rc = check_dropout(desc)) return rc;
    if (drop == nullptr) return FLARE_ERR_INVALID_ARG;
    if (int rc = check_drop(drop)) return rc;
    const size_t t = size_of(desc->dtype), r = size_of(desc->residual_dtype);
    if ((desc->rows > 0 && (!dy || !dx)) || !natural(dy, r) || !natural(dx, t)) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    if (desc->rows == 0) return FLARE_OK;
    DropoutArgs a{};
    a.x = dy; a.y = dx;
    a.ld_x = (uint32_t)(desc->stride_y ? desc->stride_y : desc->width); a.ld_y = (uint32_t)(desc->stride_x ? desc->stride_x : desc->width);
    a.rows = (uint32_t)desc->rows; a.C = (uint32_t)desc->width; a.drop = drop_args(drop);
    const bool vec = desc->width % 8 == 0 && rows16(dy, a.ld_x, r) && rows16(dx, a.ld_y, t);
    return FLARE_TWO_TYPES(desc->residual_dtype, desc->dtype, launch_dropout)(a, vec, reinterpret_cast<cudaStream_t>(stream));
}

int flare_embed_forward(const flare_embed_desc_t *desc, const flare_drop_t *drop, const void *tokens, const void *table, const void *positions, void *y,
                        flare_stream_t stream) {
    if (int rc = check_embed(desc)) return rc;
    if (int rc = check_drop(drop)) return rc;
    const size_t t = size_of(desc->dtype), o = size_of(desc->out_dtype);
    if (!table || (positions != nullptr) != (desc->positions > 0) || (desc->rows > 0 && (!tokens || !y))) return FLARE_ERR_INVALID_ARG;
    if (!natural(tokens, desc->token_bits / 8) || !natural(table, t) || !natural(positions, t) || !natural(y, o)) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    if (desc->rows == 0) return FLARE_OK;
    EmbedArgs a{};
    a.tokens = tokens; a.table = table; a.positions = positions; a.y = y;
    a.ld_t = (uint32_t)(desc->stride_table ? desc->stride_table : desc->width); a.ld_y = (uint32_t)(desc->stride_out ? desc->stride_out : desc->width);
    a.rows = (uint32_t)desc->rows; a.C = (uint32_t)desc->width; a.L = (uint32_t)std::max<int64_t>(1, desc->positions);
    a.vocab = (uint32_t)desc->vocab; a.scale = desc->scale; a.drop = drop_args(drop); a.wide = desc->token_bits == 64;
    const bool vec = desc->width % 8 == 0 && rows16(table, a.ld_t, t) && rows16(y, a.ld_y, o) && aligned16(positions);
    return FLARE_TWO_TYPES(desc->dtype, desc->out_dtype, launch_embed)(a, vec, reinterpret_cast<cudaStream_t>(stream));
}

size_t flare_embed_workspace_bytes(const flare_embed_desc_t *desc) {
    if (check_embed(desc) != FLARE_OK) return 0;
    // (whether two groups can be taken at a time is known with the tensors' addresses)
    const int sms = device_info().sms;
    return std::max(embed_layout(desc, sms, false).total, embed_layout(desc, sms, sum_in_twos(desc, sms)).total);
}

int flare_embed_backward(const flare_embed_desc_t *desc, const flare_drop_t *drop, const void *tokens, const void *dy, void *dtable, void *dpositions, int32_t accumulate,
                         void *workspace, size_t workspace_bytes, flare_stream_t stream) {
    if (int rc = check_embed(desc)) return rc;
    if (int rc = check_drop(drop)) return rc;
    const size_t t = size_of(desc->dtype), o = size_of(desc->out_dtype);
    if ((dpositions != nullptr && desc->positions == 0) || (desc->rows > 0 && (!tokens || !dy)) || !workspace || !aligned16(workspace)) return FLARE_ERR_INVALID_ARG;
    if (!natural(tokens, desc->token_bits / 8) || !natural(dy, o) || !natural(dtable, t) || !natural(dpositions, t)) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    const int sms = device_info().sms;
    if (workspace_bytes < flare_embed_workspace_bytes(desc)) return FLARE_ERR_WORKSPACE_TOO_SMALL;
    const uint32_t ld_dy = (uint32_t)(desc->stride_out ? desc->stride_out : desc->width);
    const bool vec = desc->width % 8 == 0 && rows16(dy, ld_dy, o) && aligned16(dtable) && aligned16(dpositions), twos = vec && sum_in_twos(desc, sms);
    const EmbedLayout w = embed_layout(desc, sms, twos);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const size_t table_bytes = (size_t)desc->vocab * desc->width * t;
    if (desc->rows == 0) {
        if (accumulate) return FLARE_OK;
        if (dtable) FLARE_CUDA(cudaMemsetAsync(dtable, 0, table_bytes, st));
        if (dpositions) FLARE_CUDA(cudaMemsetAsync(dpositions, 0, (size_t)desc->positions * desc->width * t, st));
        return FLARE_OK;
    }
    char *ws = static_cast<char *>(workspace);
    SumArgs a{};
    ZeroArgs z{};
    const SumShape shape = sum_shape(desc, twos);
    a.dy = dy; a.ld_dy = ld_dy;
    a.C = (uint32_t)desc->width; a.columns = (a.C + 7) / 8 * 8; a.drop = drop_args(drop);
    a.threads = shape.threads; a.lanes = shape.lanes; a.tiles = shape.tiles; a.chunks = shape.chunks;
    if ((uint64_t)(w.spans[0] + w.spans[1]) * a.tiles > ((1ull << 31) - 1)) return FLARE_ERR_UNSUPPORTED;
    const long batch = desc->positions > 0 ? desc->rows / desc->positions : 1;
    const bool whole_positions = chunk_rows_of_positions(desc, sms) % batch == 0;      // no position's rows reach over a chunk's end
    if (dtable) {
        SortArgs s{};
        s.tokens = tokens; s.wide = desc->token_bits == 64; s.rows = (uint32_t)desc->rows; s.vocab = (uint32_t)desc->vocab;
        for (int i = 0; i < 2; ++i) s.pairs[i] = reinterpret_cast<uint2 *>(ws + w.pairs[i]);
        int bits = 1;
        while (bits < 32 && (uint64_t)desc->vocab >> bits) ++bits;            // keys 0 .. vocab
        s.passes = (bits + kSortBits - 1) / kSortBits;
        s.bits = (bits + s.passes - 1) / s.passes;
        if (int rc = launch_sort(s, st)) return rc;
        if (!accumulate) {
            const uint32_t groups = (s.vocab + 31) / 32;
            z = ZeroArgs{s.pairs[sorted_in(s.passes)], s.rows, s.vocab, 0, groups, (uint64_t)desc->width * t, static_cast<uint8_t *>(dtable)};
            // (16 MB and more: some 5 us of writing)
            a.beside_zero = table_bytes >= (16u << 20) ? 2 : 1;
        }
        SumTask &k = a.task[0];
        k.pairs = s.pairs[sorted_in(s.passes)];
        k.items = s.rows; k.most = (uint32_t)desc->vocab; k.out = dtable; k.scale = desc->scale * a.drop.keep; k.add = accumulate != 0;
        k.part = reinterpret_cast<float *>(ws + w.part[0]);
        k.T = (uint32_t)chunk_rows(desc, sms); k.spans = (uint32_t)w.spans[0];
    }
    if (dpositions) {
        SumTask &k = a.task[1];
        k.items = (uint32_t)desc->rows; k.L = (uint32_t)desc->positions; k.batch = k.items / k.L; k.most = ~0u;
        k.out = dpositions; k.scale = a.drop.keep; k.add = accumulate != 0;
        k.part = reinterpret_cast<float *>(ws + w.part[1]);
        k.T = (uint32_t)chunk_rows_of_positions(desc, sms); k.spans = (uint32_t)w.spans[1];
    }
    if (!dtable && !dpositions) return FLARE_OK;
    return FLARE_TWO_TYPES(desc->out_dtype, desc->dtype, launch_sums)(a, z, vec ? (twos ? 2 : 1) : 0, whole_positions, st);
}

}  // extern "C"
