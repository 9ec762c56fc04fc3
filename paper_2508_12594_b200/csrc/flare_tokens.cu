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
    a.seed = d->seed; a.offset = d->offset; a.step = d->step;
    return a;
}
// Blocks of a kernel that walks over `items`: a thread an item, or sixteen blocks an SM (up to four of them at a time).
unsigned walk_blocks(uint64_t items, int per_block) { return (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((items + per_block - 1) / per_block, 16ull * device_info().sms)); }

int check_dropout(const flare_dropout_desc_t *d) {
    if (d == nullptr || d->rows < 0 || d->width <= 0) return FLARE_ERR_INVALID_ARG;
    for (int64_t s : {d->stride_x, d->stride_residual, d->stride_y})
        if (s != 0 && s < d->width) return FLARE_ERR_INVALID_ARG;
    if (!a_type(d->dtype) || (d->residual_dtype != d->dtype && d->residual_dtype != FLARE_DTYPE_F32)) return FLARE_ERR_UNSUPPORTED;
    return d->rows > ((int64_t)1 << 31) - 1 ? FLARE_ERR_UNSUPPORTED : FLARE_OK;
}

template <typename X, typename R>
int launch_dropout(const DropoutArgs &a, bool vec, cudaStream_t st) {
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
    if (!a_type(d->dtype) || !a_type(d->out_dtype)) return FLARE_ERR_UNSUPPORTED;
    if (d->dtype != d->out_dtype && d->dtype != FLARE_DTYPE_F32 && d->out_dtype != FLARE_DTYPE_F32) return FLARE_ERR_UNSUPPORTED;
    return d->rows > ((int64_t)1 << 31) - 1 || d->width > (1 << 20) ? FLARE_ERR_UNSUPPORTED : FLARE_OK;
}

template <typename T, typename O>
int launch_embed(const EmbedArgs &a, bool vec, cudaStream_t st) {
    if (vec) FLARE_CUDA(launch_after(embed_kernel<T, O, true>, walk_blocks((uint64_t)a.rows * (a.C / 8), kTokenThreads), kTokenThreads, 0, st, a));
    else FLARE_CUDA(launch_after(embed_kernel<T, O, false>, walk_blocks((uint64_t)a.rows * ((a.C + 255) / 256), kTokenThreads / 32), kTokenThreads, 0, st, a));
    return FLARE_OK;
}

// Rows of a chunk of the backward's sums: such that there are some 1024 threads an SM, 8 to 64.
int chunk_rows(const flare_embed_desc_t *d, int sms) {
    const long groups = (d->width + 7) / 8, want = d->rows * groups / (1024L * sms);
    return (int)std::min(64L, std::max(8L, want / 4 * 4));
}
struct EmbedLayout { size_t key[2], index[2], part[2], total; long chunks; };
EmbedLayout embed_layout(const flare_embed_desc_t *d, int sms) {
    EmbedLayout w{};
    size_t off = kHeaderBytes;
    for (int i = 0; i < 2; ++i) {
        w.key[i] = off; off += align_up(sizeof(uint32_t) * (size_t)d->rows);
        w.index[i] = off; off += align_up(sizeof(uint32_t) * (size_t)d->rows);
    }
    const int T = chunk_rows(d, sms);
    w.chunks = (d->rows + T - 1) / T;
    for (int i = 0; i < 2; ++i) {
        w.part[i] = off;
        if (i == 0 || d->positions > 0) off += align_up(sizeof(float) * 2 * (size_t)w.chunks * ((d->width + 7) / 8 * 8));
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
constexpr size_t kSortSmem = sizeof(uint32_t) * ((33u << kSortBits) + 32);

int launch_sort(SortArgs s, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    if (int rc = ensure_big_smem(embed_sort_kernel, opt_in, (int)kSortSmem)) return rc;
    int bits = 1;
    while (bits < 32 && (uint64_t)s.vocab >> bits) ++bits;    // keys 0 .. vocab
    s.passes = (bits + kSortBits - 1) / kSortBits;
    s.bits = (bits + s.passes - 1) / s.passes;
    const int n = sort_cluster(kSortSmem);
    // clusters beside the one that sorts, for what there is to set to zero: 64 KB a block and turn
    const long others = s.zeros > 0 || s.heads || s.tails ? std::min<long>((long)(s.zeros / (4096L * n)) + 1, device_info().sms / n) : 0;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = n; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(n * (1 + others)));
    cfg.blockDim = kSortThreads; cfg.dynamicSmemBytes = sizeof(uint32_t) * ((33u << s.bits) + 32); cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, embed_sort_kernel, s));
    return FLARE_OK;
}

// dy's type first
template <typename O, typename T>
int launch_sums(const SumArgs &a, bool vec, cudaStream_t st) {
    const unsigned blocks = a.task[0].blocks + a.task[1].blocks, chunks = a.task[0].chunks + a.task[1].chunks;
    if (vec) {
        FLARE_CUDA(launch_after(embed_sum_kernel<O, T, true>, blocks, kTokenThreads, 0, st, a));
        FLARE_CUDA(launch_after(embed_join_kernel<T, true>, chunks, kTokenThreads, 0, st, a));
    } else {
        FLARE_CUDA(launch_after(embed_sum_kernel<O, T, false>, blocks, kTokenThreads, 0, st, a));
        FLARE_CUDA(launch_after(embed_join_kernel<T, false>, chunks, kTokenThreads, 0, st, a));
    }
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
    auto ld = [&](int64_t s) { return (long)(s ? s : desc->width); };
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
    a.ld_x = desc->stride_y ? desc->stride_y : desc->width; a.ld_y = desc->stride_x ? desc->stride_x : desc->width;
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
    a.ld_t = desc->stride_table ? desc->stride_table : desc->width; a.ld_y = desc->stride_out ? desc->stride_out : desc->width;
    a.rows = (uint32_t)desc->rows; a.C = (uint32_t)desc->width; a.L = (uint32_t)std::max<int64_t>(1, desc->positions);
    a.vocab = desc->vocab; a.scale = desc->scale; a.drop = drop_args(drop); a.wide = desc->token_bits == 64;
    const bool vec = desc->width % 8 == 0 && rows16(table, a.ld_t, t) && rows16(y, a.ld_y, o) && aligned16(positions);
    return FLARE_TWO_TYPES(desc->dtype, desc->out_dtype, launch_embed)(a, vec, reinterpret_cast<cudaStream_t>(stream));
}

size_t flare_embed_workspace_bytes(const flare_embed_desc_t *desc) {
    return check_embed(desc) == FLARE_OK ? embed_layout(desc, device_info().sms).total : 0;
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
    const EmbedLayout w = embed_layout(desc, sms);
    if (workspace_bytes < w.total) return FLARE_ERR_WORKSPACE_TOO_SMALL;
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
    a.dy = dy; a.ld_dy = desc->stride_out ? desc->stride_out : desc->width;
    a.C = (uint32_t)desc->width; a.columns = (a.C + 7) / 8 * 8; a.T = (uint32_t)chunk_rows(desc, sms); a.drop = drop_args(drop);
    const uint64_t threads = (uint64_t)w.chunks * (a.columns / 8), blocks = (threads + kTokenThreads - 1) / kTokenThreads;
    if (2 * blocks > ((1ull << 31) - 1)) return FLARE_ERR_UNSUPPORTED;
    if (dtable) {
        SortArgs s{};
        s.tokens = tokens; s.wide = desc->token_bits == 64; s.rows = (uint32_t)desc->rows; s.vocab = desc->vocab;
        for (int i = 0; i < 2; ++i) {
            s.key[i] = reinterpret_cast<uint32_t *>(ws + w.key[i]);
            s.index[i] = reinterpret_cast<uint32_t *>(ws + w.index[i]);
        }
        if (!accumulate) {
            uint8_t *p = static_cast<uint8_t *>(dtable);
            s.heads = (uint32_t)std::min<size_t>(table_bytes, -reinterpret_cast<uintptr_t>(p) & 15u);
            s.head = p;
            s.zero = reinterpret_cast<uint4 *>(p + s.heads);
            s.zeros = (table_bytes - s.heads) / 16;
            s.tail = p + s.heads + s.zeros * 16;
            s.tails = (uint32_t)(table_bytes - s.heads - s.zeros * 16);
        }
        if (int rc = launch_sort(s, st)) return rc;
        int bits = 1;
        while (bits < 32 && (uint64_t)desc->vocab >> bits) ++bits;
        const int in = sorted_in((bits + kSortBits - 1) / kSortBits);
        SumTask &k = a.task[0];
        k.key = s.key[in]; k.index = s.index[in];
        k.items = s.rows; k.most = (uint32_t)desc->vocab; k.out = dtable; k.ld_out = desc->width; k.scale = desc->scale; k.add = accumulate != 0;
        k.part = reinterpret_cast<float *>(ws + w.part[0]);
        k.chunks = (uint32_t)w.chunks; k.blocks = (uint32_t)blocks;
    }
    if (dpositions) {
        SumTask &k = a.task[1];
        k.items = (uint32_t)desc->rows; k.L = (uint32_t)desc->positions; k.batch = k.items / k.L; k.most = ~0u;
        k.out = dpositions; k.ld_out = desc->width; k.scale = 1.f; k.add = accumulate != 0;
        k.part = reinterpret_cast<float *>(ws + w.part[1]);
        k.chunks = (uint32_t)w.chunks; k.blocks = (uint32_t)blocks;
    }
    if (!dtable && !dpositions) return FLARE_OK;
    const bool vec = desc->width % 8 == 0 && rows16(dy, a.ld_dy, o) && aligned16(dtable) && aligned16(dpositions);
    return FLARE_TWO_TYPES(desc->out_dtype, desc->dtype, launch_sums)(a, vec, st);
}

}  // extern "C"
