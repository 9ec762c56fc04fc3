// The loss over a vocabulary: argument checks, plan, workspace, launches.
#include "flare_host.h"
#include "flare_loss.cuh"

namespace flare {
namespace {

size_t size_of(int dtype) { return dtype == FLARE_DTYPE_F32 ? 4 : 2; }
bool natural(const void *p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

int need_device() {
    const DeviceView di = device_info();
    if (di.checked == -2) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "no CUDA device");
        return FLARE_ERR_CUDA;
    }
    return di.checked == 1 ? FLARE_OK : FLARE_ERR_ARCH;
}

int check_loss(const flare_loss_desc_t *d) {
    if (d == nullptr || d->rows < 0 || d->width <= 0 || d->vocab <= 0) return FLARE_ERR_INVALID_ARG;
    if (d->label_bits != 32 && d->label_bits != 64) return FLARE_ERR_INVALID_ARG;
    if (!(d->scale > 0.f) || !std::isfinite(d->scale) || !std::isfinite(d->dloss_scale)) return FLARE_ERR_INVALID_ARG;
    for (int64_t s : {d->stride_x, d->stride_w, d->stride_dx, d->stride_dw})
        if (s != 0 && s < d->width) return FLARE_ERR_INVALID_ARG;
    if (d->dtype != FLARE_DTYPE_F32 && d->dtype != FLARE_DTYPE_BF16 && d->dtype != FLARE_DTYPE_F16) return FLARE_ERR_UNSUPPORTED;
    return d->rows > (1 << 30) || d->width > 16384 || d->vocab > (1 << 28) ? FLARE_ERR_UNSUPPORTED : FLARE_OK;
}

// G of a piece of the vocabulary takes this much scratch (or 256 words of it where that is more).  A piece costs three launches, their ends, and another pass over the sums of dX: 16384 rows over 50021 words of
// 512 take 3.2 ms in pieces of 256 MB, 2.83 of 512, 2.97 of 1024; 18944 over 50021 of 256 take 2.34, 2.06, 1.97; 8192 over 128256 of 1024 take 6.6 in each.
constexpr size_t kPieceBytes = 512u << 20;
struct LossPlan {
    bool bf16;                   // what is multiplied is bfloat16 (else float16)
    int planes, g_planes;        // values of 16 bits to an element of X and W, of G
    int Cp, chunks, x_blocks, pairs;
    long cap;
    int width;                   // of a tile of X W^T
    int Vp, pieces;              // words of a piece
    int grad_width, tiles_c;
};
// Columns of a tile of X W^T.  Tiles of 128 take some 0.6 of the time of one of 256 (they read as many rows), which pays where they fill the last
// round of pairs better: 1000 rows over 5000 words of 256, forward and backward, 60.7 us, with 256 columns 62.3; forward of 256 rows over 32000 words of 1024 28.0 us, with 256 columns 19.2.
int tile_width(long row_tiles, long words, int pairs) {
    const long wide = row_tiles * ((words + 255) / 256), narrow = row_tiles * ((words + 127) / 128);
    return 0.6 * (double)((narrow + pairs - 1) / pairs) < (double)((wide + pairs - 1) / pairs) ? 128 : 256;
}
LossPlan loss_plan(const flare_loss_desc_t *d, int sms, bool backward) {
    LossPlan p{};
    const bool f32 = d->dtype == FLARE_DTYPE_F32;
    // G in one 16-bit value is off by 2^-9 (2^-12): gradients by 1.06 times what rounding exact ones gives, 1.3 to 1.45 times where every row has its own dloss, or of few words, where a label's p is not next to 0; of few
    // rows, whose rounding does not average out, up to 1.76 times.  In two values they are as good as rounded exact ones, for twice the products of the gradients and G's bytes: bfloat16, 131072 rows over 256 words,
    // C = 128: 153 us a step (one value: 112); 2000 over 4096, C = 1024: 118 (93); 8192 over 8000, C = 512: 385 (266); 16384 over 32000, C = 128: 1466 (892); 64 over 32000, C = 1024: 146 (111).  So of one tile of
    // rows, and of vocabularies where it is a third or less, as if W were small.
    const bool two = !f32 && backward && (d->rows <= 256 || (d->vocab <= 8192 && (long)d->vocab * d->width <= (4L << 20)));
    p.bf16 = d->dtype != FLARE_DTYPE_F16;
    p.planes = f32 ? 3 : 1;
    p.g_planes = f32 ? 3 : two ? 2 : 1;
    // rows of packed X and W: whole 16 bytes, of wide ones whole lines (TMA takes 128-byte pieces of them)
    p.Cp = d->width > 256 ? (d->width + 63) / 64 * 64 : (d->width + 7) / 8 * 8;
    p.chunks = (int)((d->rows + kLossChunk - 1) / kLossChunk);
    p.x_blocks = d->dtype == FLARE_DTYPE_F16 && backward ? (int)std::max(1L, std::min(4L * sms, (long)d->rows * d->width / 8192)) : 0;
    p.pairs = std::max(1, sms / 2);
    p.cap = std::max(1L, (long)(d->rows + 255) / 256) * 256;
    p.width = tile_width(p.cap / 256, d->vocab, p.pairs);
    const long words = ((long)d->vocab + 255) / 256 * 256, most = std::max(256L, (long)(kPieceBytes / (2 * p.g_planes * p.cap)) / 256 * 256);
    p.pieces = (int)((words + most - 1) / most);
    p.Vp = (int)((words / 256 + p.pieces - 1) / p.pieces * 256);
    p.pieces = (int)((words + p.Vp - 1) / p.Vp);
    // (a width that 256 does not divide well is worked off in 128s, which take 0.6 each: 8192 rows over 32000 words, C = 128: 502 us, with 256 columns 517; C = 256: 726, with 256 columns 622)
    p.grad_width = 1.2 * ((d->width + 127) / 128) < 2.0 * ((d->width + 255) / 256) ? 128 : 256;
    p.tiles_c = (d->width + p.grad_width - 1) / p.grad_width;
    return p;
}
// Forward of up to eight rows (loss_few_kernel): rows it is compiled for, or 0 where X would not fit beside a second block of an SM.
int few_rows(const flare_loss_desc_t *d) {
    const int R = d->rows <= 1 ? 1 : d->rows <= 2 ? 2 : d->rows <= 4 ? 4 : 8;
    return d->rows <= 8 && few_smem(R, d->width) <= 96 * 1024 ? R : 0;
}
int few_blocks(const flare_loss_desc_t *d, long words, int sms) {
    // rounds of equal size over the warps that are at work at a time
    const long groups = (words + kFewWords - 1) / kFewWords, warps = (long)sms * (few_rows(d) <= 2 ? 4 : 2) * (kFewThreads / 32), rounds = (groups + warps - 1) / warps;
    return (int)(((groups + rounds - 1) / rounds + kFewThreads / 32 - 1) / (kFewThreads / 32));
}
struct LossLayout { size_t info, rank, chunk, largest, px, pd, pw, index, label, part, chosen, gave_up, lse_of, gm, coef, g, acc, slots, total; };
// What is taken as it stands and needs no place for a packed copy: W of 16 bits, and X of few rows or of a small vocabulary in the forward, on 16-byte boundaries.
struct LossLies { bool w, x; };
long row_stride(int64_t stride, int width) { return stride ? stride : width; }
LossLies loss_lies(const flare_loss_desc_t *d, bool backward, bool x_aligned, bool w_aligned) {
    if (d->dtype == FLARE_DTYPE_F32) return LossLies{false, false};
    const bool w = w_aligned && row_stride(d->stride_w, d->width) % 8 == 0, x = x_aligned && row_stride(d->stride_x, d->width) % 8 == 0;
    // X too without packing, where all rows are one tile's (64 rows over 32000 words of 1024 take 20.3 us, packed 24.4) or the vocabulary is so small that another pass over X costs more than most rows without a label
    // do, whose share is known to the device alone: 131072 rows over 256 words of 128 take 22.9 us whatever it is, packed 30.1 with 0.1 of them, 25.4 with 0.3, 21.9 with 0.5, 17.4 with 0.85; 20000 over 1000 of 512
    // 21.1 and 30.4, 27.1, 26.0, 19.9
    return LossLies{w, !backward && w && x && (d->rows <= 256 || d->vocab <= 2048)};
}
// Rows that loss_few_kernel is run for, 0: it is not.  (Five to eight rows that need no packing are done sooner by the tensor cores: 8 rows over 32000 words of 1024 in bfloat16 in 23 us instead of 32.6, where four take
// 25.7 and 22.0, two 23.7 and 20.2, one 26.2 and 16.5; of 1001, which are packed, eight take 54 and 36.6; in float32, of 2048, 240 and 73.)
int few_rows_of(const flare_loss_desc_t *d, LossLies lies) { return lies.x && d->rows > 4 ? 0 : few_rows(d); }
LossLayout loss_layout(const flare_loss_desc_t *d, const LossPlan &p, bool backward, LossLies lies) {
    const bool few = !backward && few_rows_of(d, lies) > 0;   // (nothing is packed)
    LossLayout w{};
    size_t off = kHeaderBytes;
    auto take = [&](size_t &at, size_t bytes) { at = off; off += align_up(bytes); };
    take(w.info, sizeof(LossInfo));
    take(w.rank, sizeof(int) * (size_t)d->rows);
    take(w.chunk, sizeof(LossChunk) * (size_t)p.chunks);
    take(w.largest, sizeof(int) * (size_t)p.x_blocks);
    const size_t row = sizeof(uint16_t) * (size_t)p.planes * p.Cp;
    take(w.px, lies.x || few ? 0 : row * p.cap);
    take(w.pw, lies.w || few ? 0 : row * d->vocab);
    take(w.index, sizeof(int) * (size_t)p.cap);
    take(w.label, sizeof(int) * (size_t)p.cap);
    if (!backward) {
        const long tiles = (d->vocab + p.width - 1) / p.width;
        take(w.part, sizeof(float2) * (few ? (size_t)few_blocks(d, d->vocab, 2 * p.pairs) : (size_t)tiles) * p.cap);
        take(w.chosen, sizeof(float) * (size_t)p.cap);
        take(w.gave_up, sizeof(uint32_t) * 2 * (size_t)p.pairs);
    } else {
        take(w.pd, p.bf16 ? 0 : row * p.cap);
        take(w.lse_of, sizeof(float) * (size_t)p.cap);
        take(w.gm, sizeof(float) * (size_t)p.cap);
        take(w.coef, sizeof(float) * (size_t)p.cap);
        take(w.g, sizeof(uint16_t) * (size_t)p.g_planes * p.cap * p.Vp);
        take(w.acc, p.pieces > 1 ? sizeof(float) * (size_t)p.cap * p.tiles_c * p.grad_width : 0);
        take(w.slots, sizeof(float) * 4 * (size_t)p.pairs * p.grad_width * 128);
    }
    w.total = off;
    return w;
}

// 16-bit elements [planes, rows, cols], rows `ld` apart, in boxes of 64 columns (128-byte swizzle).
int make_plane_map(CUtensorMap *m, const void *base, bool bf16, long cols, long rows, long planes, long ld, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled not available");
        return FLARE_ERR_CUDA;
    }
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)(planes > 1 ? rows : 1)};   // (of one plane the distance to the next is never used, but has a limit)
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
    const CUresult r = fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled(loss) failed: %d", (int)r);
        return FLARE_ERR_CUDA;
    }
    return FLARE_OK;
}

template <int kKind, int kF, int kG, typename E>
int launch_loss(const LossMaps &maps, const LossArgs &a, int pairs, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    auto *kernel = loss_kernel<kKind, kF, kG, E>;
    if (int rc = ensure_big_smem(kernel, opt_in, (int)kLossSmem)) return rc;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * (unsigned)pairs);
    cfg.blockDim = kLossThreads; cfg.dynamicSmemBytes = kLossSmem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, kernel, maps, a));
    return FLARE_OK;
}

int launch_merge(const LossMerge &m, long rows, cudaStream_t st) {
    const int warps = std::min(kMergeWarps, std::max(1, m.parts / 4));
    FLARE_CUDA(launch_after(loss_merge_kernel, (unsigned)std::min<long>((rows + 31) / 32, 65535L), 32 * warps, 0, st, m));
    return FLARE_OK;
}

template <typename T>
int launch_pack(const LossPack &k, int blocks, cudaStream_t st) {
    FLARE_CUDA(launch_after(loss_pack_kernel<T>, (unsigned)blocks, kPackThreads, 0, st, k));
    return FLARE_OK;
}

template <typename T, int R, bool kVec, int kG>
int launch_few_as(const LossFew &f, int blocks, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    auto *kernel = loss_few_kernel<T, R, kVec, kG>;
    if (int rc = ensure_big_smem(kernel, opt_in, 96 * 1024)) return rc;
    FLARE_CUDA(launch_after(kernel, (unsigned)blocks, kFewThreads, few_smem(R, f.C), st, f));
    return FLARE_OK;
}
template <typename T, int kG>
int launch_few_of(const LossFew &f, int R, int blocks, cudaStream_t st) {
    const bool vec = f.C % 8 == 0 && aligned16(f.w) && f.ld_w * (long)sizeof(T) % 16 == 0;
    auto launch = R == 1   ? (vec ? launch_few_as<T, 1, true, kG> : launch_few_as<T, 1, false, kG>)
                  : R == 2 ? (vec ? launch_few_as<T, 2, true, kG> : launch_few_as<T, 2, false, kG>)
                  : R == 4 ? (vec ? launch_few_as<T, 4, true, kG> : launch_few_as<T, 4, false, kG>)
                           : (vec ? launch_few_as<T, 8, true, kG> : launch_few_as<T, 8, false, kG>);
    return launch(f, blocks, st);
}
// (G of few rows is three or two values: loss_plan)
int launch_few(const LossFew &f, int dtype, bool backward, int R, int blocks, cudaStream_t st) {
    auto launch = dtype == FLARE_DTYPE_F32    ? (backward ? launch_few_of<float, 3> : launch_few_of<float, 0>)
                  : dtype == FLARE_DTYPE_BF16 ? (backward ? launch_few_of<__nv_bfloat16, 2> : launch_few_of<__nv_bfloat16, 0>)
                                              : (backward ? launch_few_of<__half, 2> : launch_few_of<__half, 0>);
    return launch(f, R, blocks, st);
}
LossFew few_args(const flare_loss_desc_t *d, const LossPlan &p, const void *x, const void *w, const void *labels) {
    LossFew f{};
    f.x = x; f.w = w; f.labels = labels; f.wide = d->label_bits == 64; f.rows = (int)d->rows; f.C = d->width; f.V = d->vocab; f.words = d->vocab;
    f.ld_x = row_stride(d->stride_x, d->width); f.ld_w = row_stride(d->stride_w, d->width); f.cap = p.cap; f.scale = d->scale;
    return f;
}

// Checks that forward and backward share.
int check_loss_call(const flare_loss_desc_t *d, const void *x, const void *w, const void *labels, void *workspace, size_t workspace_bytes, bool backward) {
    const size_t t = size_of(d->dtype);
    if (!workspace || !aligned16(workspace) || !w || (d->rows > 0 && (!x || !labels))) return FLARE_ERR_INVALID_ARG;
    if (!natural(x, t) || !natural(w, t) || !natural(labels, d->label_bits / 8)) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    return workspace_bytes < loss_layout(d, loss_plan(d, device_info().sms, backward), backward, loss_lies(d, backward, aligned16(x), aligned16(w))).total ? FLARE_ERR_WORKSPACE_TOO_SMALL : FLARE_OK;
}

// Scan and packing, and the maps of X and W; what only the backward has is in k already.
int prepare_loss(const flare_loss_desc_t *d, const LossPlan &p, const LossLayout &l, LossLies lies, char *ws, const void *x, const void *w, const void *labels, LossPack k, LossMaps *maps,
                 LossArgs *a, cudaStream_t st) {
    const bool f32 = d->dtype == FLARE_DTYPE_F32, bf16 = p.bf16;
    const long ld_x = row_stride(d->stride_x, d->width), ld_w = row_stride(d->stride_w, d->width);
    const bool own_w = !lies.w;
    LossScan s{};
    s.labels = labels; s.wide = d->label_bits == 64; s.rows = d->rows; s.V = d->vocab; s.chunks = p.chunks;
    if (k.pd) {
        s.C = d->width; s.x_blocks = p.x_blocks; s.x = x; s.ld_x = ld_x; s.dloss = k.dloss;
        s.largest = reinterpret_cast<int *>(ws + l.largest);
    }
    s.rank = reinterpret_cast<int *>(ws + l.rank); s.chunk = reinterpret_cast<LossChunk *>(ws + l.chunk);
    s.status = reinterpret_cast<uint32_t *>(ws);
    int rc;
    // rows of a block: so many that a thread has four groups of columns, and that there are no more than four blocks an SM; whole parts of a chunk
    k.pack_rows = 4;
    while (k.pack_rows < kLossChunk && ((long)k.pack_rows * (p.Cp / 8) < 4 * kPackThreads || (long)k.pack_rows * 4 * device_info().sms < d->rows)) k.pack_rows *= 2;
    const bool alone = d->rows <= kPackAlone && !k.pd && k.pack_rows <= kPackThreads;
    if (!alone) FLARE_CUDA(launch_after(loss_scan_kernel, (unsigned)(s.chunks + s.x_blocks), kScanThreads, 0, st, s));
    k.labels = labels; k.x = x; k.w = w; k.wide = s.wide; k.rows = d->rows; k.cap = p.cap; k.ld_x = ld_x; k.ld_w = ld_w;
    k.w_rows = own_w ? d->vocab : 0; k.C = d->width; k.Cp = p.Cp; k.V = d->vocab; k.chunks = p.chunks;
    k.pack_blocks = (int)((d->rows + k.pack_rows - 1) / k.pack_rows);
    k.rank = alone ? nullptr : s.rank; k.status = s.status; k.chunk = s.chunk; k.largest = s.largest; k.x_blocks = s.x_blocks;
    k.info = reinterpret_cast<LossInfo *>(ws + l.info);
    k.px = reinterpret_cast<uint16_t *>(ws + l.px); k.pw = reinterpret_cast<uint16_t *>(ws + l.pw);
    k.index = reinterpret_cast<int *>(ws + l.index); k.label = reinterpret_cast<int *>(ws + l.label);
    const int blocks = k.pack_blocks + (int)std::min<long>((k.w_rows * (p.Cp / 8) + 4 * kPackThreads - 1) / (4 * kPackThreads), 16L * device_info().sms);
    if ((rc = f32 ? launch_pack<float>(k, blocks, st) : d->dtype == FLARE_DTYPE_F16 ? launch_pack<__half>(k, blocks, st) : launch_pack<__nv_bfloat16>(k, blocks, st)) != FLARE_OK) return rc;
    if ((rc = make_plane_map(&maps->x, k.px, bf16, p.Cp, p.cap, p.planes, p.Cp, 64)) != FLARE_OK) return rc;
    if ((rc = own_w ? make_plane_map(&maps->w, k.pw, bf16, p.Cp, d->vocab, p.planes, p.Cp, 64)
                    : make_plane_map(&maps->w, w, bf16, d->width, d->vocab, 1, ld_w, 64)) != FLARE_OK)
        return rc;
    a->info = k.info; a->status = s.status; a->C = d->width; a->V = d->vocab; a->bf16 = bf16; a->cap = p.cap; a->scale = d->scale;
    a->label = k.label; a->index = k.index;
    return FLARE_OK;
}

}  // namespace
}  // namespace flare

using namespace flare;

extern "C" {

size_t flare_loss_workspace_bytes(const flare_loss_desc_t *desc, int32_t backward) {
    if (check_loss(desc) != FLARE_OK) return 0;
    const bool back = (backward & ~FLARE_LOSS_ALIGNED) != 0;
    const LossPlan p = loss_plan(desc, device_info().sms, back);
    auto bytes = [&](bool x, bool w) { return loss_layout(desc, p, back, loss_lies(desc, back, x, w)).total; };
    if (backward & FLARE_LOSS_ALIGNED) return bytes(true, true);
    return std::max(bytes(true, true), std::max(bytes(false, true), std::max(bytes(true, false), bytes(false, false))));
}

int flare_loss_forward(const flare_loss_desc_t *desc, const void *x, const void *w, const void *labels, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                       flare_stream_t stream) {
    if (int rc = check_loss(desc)) return rc;
    if (desc->rows > 0 && (!loss || !lse || !natural(loss, 4) || !natural(lse, 4))) return FLARE_ERR_INVALID_ARG;
    if (int rc = check_loss_call(desc, x, w, labels, workspace, workspace_bytes, false)) return rc;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (desc->rows == 0) {
        FLARE_CUDA(cudaMemsetAsync(workspace, 0, kHeaderBytes, st));
        return FLARE_OK;
    }
    const LossPlan p = loss_plan(desc, device_info().sms, false);
    const LossLies lies = loss_lies(desc, false, aligned16(x), aligned16(w));
    const LossLayout l = loss_layout(desc, p, false, lies);
    char *ws = static_cast<char *>(workspace);
    const long ld_x = row_stride(desc->stride_x, desc->width), ld_w = row_stride(desc->stride_w, desc->width);
    const bool direct = lies.x;
    const int R = few_rows_of(desc, lies);
    if (R) {
        LossFew f = few_args(desc, p, x, w, labels);
        f.part = reinterpret_cast<float2 *>(ws + l.part); f.chosen = reinterpret_cast<float *>(ws + l.chosen);
        const int blocks = few_blocks(desc, desc->vocab, 2 * p.pairs);
        if (int rc = launch_few(f, desc->dtype, false, R, blocks, st)) return rc;
        LossMerge m{};
        m.part = f.part; m.chosen = f.chosen; m.cap = p.cap; m.parts = blocks; m.loss = loss; m.lse = lse;
        m.labels = labels; m.wide = f.wide; m.V = f.V; m.direct = f.rows; m.status = reinterpret_cast<uint32_t *>(ws); m.scale = desc->scale;
        return launch_merge(m, desc->rows, st);
    }
    LossPack k{};
    k.loss = loss; k.lse = lse;
    LossMaps maps{};
    LossArgs a{};
    if (direct) {
        const bool bf16 = desc->dtype == FLARE_DTYPE_BF16;
        int rc;
        if ((rc = make_plane_map(&maps.x, x, bf16, desc->width, desc->rows, 1, ld_x, 64)) != FLARE_OK) return rc;
        if ((rc = make_plane_map(&maps.w, w, bf16, desc->width, desc->vocab, 1, ld_w, 64)) != FLARE_OK) return rc;
        a.C = desc->width; a.V = desc->vocab; a.bf16 = bf16; a.cap = p.cap; a.scale = desc->scale; a.status = reinterpret_cast<uint32_t *>(ws);
        a.labels = labels; a.wide = desc->label_bits == 64; a.direct = (int)desc->rows; a.gave_up = reinterpret_cast<uint32_t *>(ws + l.gave_up);
    } else if (int rc = prepare_loss(desc, p, l, lies, ws, x, w, labels, k, &maps, &a, st)) {
        return rc;
    }
    a.words = desc->vocab; a.width = p.width; a.tiles_v = (desc->vocab + p.width - 1) / p.width;
    a.part = reinterpret_cast<float2 *>(ws + l.part); a.chosen = reinterpret_cast<float *>(ws + l.chosen);
    if (a.tiles_v == 1 && !direct) { a.loss = loss; a.lse = lse; }
    const int pairs = (int)std::min<long>(p.pairs, p.cap / 256 * a.tiles_v);
    // (products of few steps, whose ends bound the tile, in turns: 37137 rows over 25943 words of 128 take 356 us instead of 444, 5003 over 10007 of 512 45.7 and 46.2)
    auto stats = p.planes == 3 ? launch_loss<kLossStats, 3, 1, float> : desc->width <= 64 * kLossDeep<kLossTurns, 1, 1> ? launch_loss<kLossTurns, 1, 1, float> : launch_loss<kLossStats, 1, 1, float>;
    if (int rc = stats(maps, a, pairs, st)) return rc;
    if (a.loss) return FLARE_OK;
    LossMerge m{};
    m.info = a.info; m.part = a.part; m.chosen = a.chosen; m.index = a.index; m.cap = p.cap; m.parts = a.tiles_v; m.loss = loss; m.lse = lse;
    m.labels = a.labels; m.wide = a.wide; m.V = a.V; m.direct = a.direct; m.gave_up = a.gave_up; m.status = a.status; m.blocks = 2 * pairs; m.scale = desc->scale;
    return launch_merge(m, desc->rows, st);
}

int flare_loss_backward(const flare_loss_desc_t *desc, const void *x, const void *w, const void *labels, const float *lse, const float *dloss, void *dx, void *dw,
                        void *workspace, size_t workspace_bytes, flare_stream_t stream) {
    if (int rc = check_loss(desc)) return rc;
    const size_t t = size_of(desc->dtype);
    if ((!dx && !dw) || (desc->rows > 0 && !lse) || !natural(lse, 4) || !natural(dloss, 4) || !natural(dx, t) || !natural(dw, t)) return FLARE_ERR_INVALID_ARG;
    if (int rc = check_loss_call(desc, x, w, labels, workspace, workspace_bytes, true)) return rc;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const long ld_dx = desc->stride_dx ? desc->stride_dx : desc->width, ld_dw = desc->stride_dw ? desc->stride_dw : desc->width;
    if (desc->rows == 0) {
        FLARE_CUDA(cudaMemsetAsync(workspace, 0, kHeaderBytes, st));
        if (dw) FLARE_CUDA(cudaMemset2DAsync(dw, ld_dw * t, 0, desc->width * t, desc->vocab, st));
        return FLARE_OK;
    }
    const LossPlan p = loss_plan(desc, device_info().sms, true);
    const LossLies lies = loss_lies(desc, true, aligned16(x), aligned16(w));
    const LossLayout l = loss_layout(desc, p, true, lies);
    const bool f32 = desc->dtype == FLARE_DTYPE_F32, bf16 = p.bf16;
    char *ws = static_cast<char *>(workspace);
    LossPack k{};
    k.lse_in = lse; k.dloss = dloss; k.mult = desc->scale * desc->dloss_scale;
    k.lse_of = reinterpret_cast<float *>(ws + l.lse_of); k.gm = reinterpret_cast<float *>(ws + l.gm); k.coef = reinterpret_cast<float *>(ws + l.coef);
    // G in bfloat16: q where one dloss is that of all rows (a label's q is next to -1, which is no rounding), else times it, for a second X would be a second rounding; in float16: q times 2^15, or times 2^14 and a row's
    // mantissa of dloss, below 2
    k.g_factor = !bf16 ? dloss ? 16384.f : 32768.f : dloss ? 0.f : 1.f;
    k.dx = dx; k.ld_dx = ld_dx;
    k.pd = bf16 || !dloss || !dw ? nullptr : reinterpret_cast<uint16_t *>(ws + l.pd);
    LossMaps maps{};
    LossArgs a{};
    if (int rc = prepare_loss(desc, p, l, lies, ws, x, w, labels, k, &maps, &a, st)) return rc;
    int rc;
    if (k.pd) {
        if ((rc = make_plane_map(&maps.d, k.pd, bf16, p.Cp, p.cap, p.planes, p.Cp, 64)) != FLARE_OK) return rc;
    } else {
        maps.d = maps.x;
    }
    if ((rc = make_plane_map(&maps.g, ws + l.g, bf16, p.Vp, p.cap, p.g_planes, p.Vp, 64)) != FLARE_OK) return rc;
    a.g = reinterpret_cast<uint16_t *>(ws + l.g); a.ld_g = p.Vp;
    a.lse_of = k.lse_of; a.gm = k.gm; a.coef = k.coef; a.grad_width = p.grad_width; a.tiles_c = p.tiles_c;
    a.dw = dw; a.dx = dx; a.ld_dw = ld_dw; a.ld_dx = ld_dx;
    auto vec = [&](const void *q, long ld) { return desc->width * t % 16 == 0 && ld * t % 16 == 0 && aligned16(q); };
    a.dw_vec = vec(dw, ld_dw); a.dx_vec = vec(dx, ld_dx);
    a.dw_factor = k.g_factor != 0.f ? k.mult / k.g_factor : 1.f;
    a.acc = reinterpret_cast<float *>(ws + l.acc); a.slots = reinterpret_cast<float *>(ws + l.slots);
    auto weights = f32 ? launch_loss<kLossWeights, 3, 3, float> : p.g_planes == 2 ? launch_loss<kLossWeights, 1, 2, float> : launch_loss<kLossWeights, 1, 1, float>;
    auto grads = f32 ? launch_loss<kLossGrads, 3, 3, float>
                 : bf16 ? (p.g_planes == 2 ? launch_loss<kLossGrads, 1, 2, __nv_bfloat16> : launch_loss<kLossGrads, 1, 1, __nv_bfloat16>)
                        : (p.g_planes == 2 ? launch_loss<kLossGrads, 1, 2, __half> : launch_loss<kLossGrads, 1, 1, __half>);
    auto *join = f32 ? loss_join_kernel<float> : desc->dtype == FLARE_DTYPE_BF16 ? loss_join_kernel<__nv_bfloat16> : loss_join_kernel<__half>;
    // few rows: G by the kernel that the forward's statistics are of
    const int R = few_rows_of(desc, loss_lies(desc, false, aligned16(x), aligned16(w)));
    LossFew few = few_args(desc, p, x, w, labels);
    few.lse_in = lse; few.gm = k.gm; few.g = a.g; few.ld_g = a.ld_g;
    // of tiles that several pairs can have shared: fewer than a round of either gradient
    const long warps = 2L * (p.pairs - 1) * 8 * (p.grad_width / kJoinCols);
    for (int i = 0; i < p.pieces; ++i) {
        a.v0 = i * p.Vp;
        a.words = std::min(p.Vp, desc->vocab - a.v0);
        a.first = i == 0; a.last = i + 1 == p.pieces;
        a.width = tile_width(p.cap / 256, a.words, p.pairs);
        a.tiles_v = (a.words + a.width - 1) / a.width;
        if (R) {
            few.v0 = a.v0; few.words = a.words;
            if ((rc = launch_few(few, desc->dtype, true, R, few_blocks(desc, a.words, 2 * p.pairs), st)) != FLARE_OK) return rc;
        } else if ((rc = weights(maps, a, (int)std::min<long>(p.pairs, p.cap / 256 * a.tiles_v), st)) != FLARE_OK) {
            return rc;
        }
        if ((rc = grads(maps, a, p.pairs, st)) != FLARE_OK) return rc;
        FLARE_CUDA(launch_after(join, (unsigned)((warps + kJoinWarps - 1) / kJoinWarps), 32 * kJoinWarps, 0, st, a, p.pairs));
    }
    return FLARE_OK;
}

}  // extern "C"
