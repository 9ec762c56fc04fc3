// Entry points of the operators around a block: argument checks, workspace, dispatch on the types.
#include "flare_block_launch.cuh"

namespace flare {
namespace {

size_t size_of(int dtype) { return dtype == FLARE_DTYPE_F32 ? 4 : 2; }

int check_block(const flare_block_desc_t *d, bool join) {
    if (d == nullptr) return FLARE_ERR_INVALID_ARG;
    if (d->rows < 0 || d->width <= 0) return FLARE_ERR_INVALID_ARG;
    if (!(d->pre_eps >= 0.f) || !(d->post_eps >= 0.f) || !std::isfinite(d->pre_eps) || !std::isfinite(d->post_eps) || !std::isfinite(d->residual_scale))
        return FLARE_ERR_INVALID_ARG;
    for (int64_t s : {d->stride_x, d->stride_branch, d->stride_gate, d->stride_y, d->stride_h, d->stride_dy, d->stride_dh, d->stride_dx, d->stride_dbranch,
                      d->stride_dgate})
        if (s != 0 && s < d->width) return FLARE_ERR_INVALID_ARG;
    auto norm = [](int n) { return n == FLARE_NORM_NONE || n == FLARE_NORM_LAYER || n == FLARE_NORM_RMS; };
    if (!norm(d->pre_norm) || !norm(d->post_norm) || d->gate < FLARE_GATE_NONE || d->gate > FLARE_GATE_LINEAR) return FLARE_ERR_INVALID_ARG;
    if (join && d->gate != FLARE_GATE_NONE && (d->gate_rows < 1 || d->rows % d->gate_rows != 0)) return FLARE_ERR_INVALID_ARG;
    if (!join && d->pre_norm == FLARE_NORM_NONE) return FLARE_ERR_INVALID_ARG;
    if (d->dtype != FLARE_DTYPE_F32 && d->dtype != FLARE_DTYPE_BF16 && d->dtype != FLARE_DTYPE_F16) return FLARE_ERR_UNSUPPORTED;
    if (d->residual_dtype != d->dtype && d->residual_dtype != FLARE_DTYPE_F32) return FLARE_ERR_UNSUPPORTED;
    if (d->width > kBlockMaxWidth || d->rows > ((int64_t)1 << 31) - 1) return FLARE_ERR_UNSUPPORTED;
    return FLARE_OK;
}

// Rows that can be moved 16 bytes at a time: every tensor that is used.
struct Aligned {
    bool ok, natural = true;                                // natural: every pointer aligned to its elements
    explicit Aligned(int C) : ok(C % 8 == 0) {}
    void add(const void *p, long ld, size_t size) {
        if (reinterpret_cast<uintptr_t>(p) % size != 0) natural = false;
        if (p != nullptr && (!aligned16(p) || ld * size % 16 != 0)) ok = false;
    }
};

BlockArgs common_args(const flare_block_desc_t *d, bool join) {
    BlockArgs a{};
    a.rows = d->rows;
    a.C = d->width;
    a.inv_c = 1.f / (float)d->width;
    auto ld = [&](int64_t s) { return (long)(s ? s : d->width); };
    a.ld_x = ld(d->stride_x); a.ld_o = ld(d->stride_branch); a.ld_g = ld(d->stride_gate); a.ld_y = ld(d->stride_y); a.ld_h = ld(d->stride_h);
    a.ld_dy = ld(d->stride_dy); a.ld_dh = ld(d->stride_dh); a.ld_dx = ld(d->stride_dx); a.ld_do = ld(d->stride_dbranch); a.ld_dg = ld(d->stride_dgate);
    a.has_pre = d->pre_norm != FLARE_NORM_NONE; a.layer_pre = d->pre_norm == FLARE_NORM_LAYER; a.eps_pre = d->pre_eps;
    a.has_post = join && d->post_norm != FLARE_NORM_NONE; a.layer_post = d->post_norm == FLARE_NORM_LAYER; a.eps_post = d->post_eps;
    a.gate = join ? d->gate : 0;
    a.grouped = a.gate && d->gate_rows > 1;
    a.group = a.grouped ? d->gate_rows : std::max<long>(d->rows, 1);
    a.alpha = join ? d->residual_scale : 1.f;
    return a;
}
bool float_params_ok(std::initializer_list<const float *> ps) {
    for (const float *p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return false;
    return true;
}

int need_device() {
    const DeviceView di = device_info();
    if (di.checked == -2) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "no CUDA device");
        return FLARE_ERR_CUDA;
    }
    return di.checked == 1 ? FLARE_OK : FLARE_ERR_ARCH;
}

#define FLARE_BLOCK_TYPES(d, call)                                                                                   \
    ((d)->dtype == FLARE_DTYPE_F32    ? call<float, float>                                                           \
     : (d)->dtype == FLARE_DTYPE_BF16 ? ((d)->residual_dtype == FLARE_DTYPE_F32 ? call<__nv_bfloat16, float> : call<__nv_bfloat16, __nv_bfloat16>) \
                                      : ((d)->residual_dtype == FLARE_DTYPE_F32 ? call<__half, float> : call<__half, __half>))

int forward(const flare_block_desc_t *d, BlockArgs a, cudaStream_t st) {
    if (int rc = need_device()) return rc;
    if (d->rows == 0) return FLARE_OK;
    const size_t t = size_of(d->dtype), r = size_of(d->residual_dtype);
    Aligned al(d->width);
    al.add(a.x, a.ld_x, r); al.add(a.o, a.ld_o, t); al.add(a.g, a.ld_g, t); al.add(a.y, a.ld_y, r); al.add(a.h, a.ld_h, t);
    if (!al.natural) return FLARE_ERR_INVALID_ARG;
    return FLARE_BLOCK_TYPES(d, block_forward)(a, al.ok, device_info().sms, st);
}

// Bytes of the partial sums, for whichever form of the kernels the tensors' alignment leads to.
size_t partial_bytes(const flare_block_desc_t *d, long group) {
    size_t bytes = 0;
    for (int vectors : {0, 1, 2}) {
        const BlockPlan p = block_plan(d->rows, group, d->width, vectors > 0, device_info().sms, std::max(vectors, 1));
        bytes = std::max(bytes, (size_t)p.groups * p.chunks * 4 * d->width * sizeof(float));
    }
    return align_up(std::max<size_t>(bytes, 1));
}
long group_of(const flare_block_desc_t *d) { return d->gate != FLARE_GATE_NONE && d->gate_rows > 1 ? d->gate_rows : std::max<long>(d->rows, 1); }

struct BlockGrads { float *d_scale, *dw_post, *db_post, *dw_pre, *db_pre; };

int backward(const flare_block_desc_t *d, bool join, BlockArgs a, const BlockGrads &out, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    if (workspace_bytes < partial_bytes(d, a.group)) return FLARE_ERR_WORKSPACE_TOO_SMALL;
    if (int rc = need_device()) return rc;
    const int sms = device_info().sms;
    const size_t t = size_of(d->dtype), r = size_of(d->residual_dtype);
    Aligned al(d->width);
    al.add(a.x, a.ld_x, r); al.add(a.dy, a.ld_dy, r); al.add(a.dx, a.ld_dx, r); al.add(a.dh, a.ld_dh, t); al.add(a.o, a.ld_o, t); al.add(a.g, a.ld_g, t);
    al.add(a.d_o, a.ld_do, t); al.add(a.dg, a.ld_dg, t);
    if (!al.natural) return FLARE_ERR_INVALID_ARG;
    const bool bias = !al.ok || a.b_post || out.db_pre || out.db_post;
    const BlockPlan plan = block_plan(d->rows, a.group, d->width, al.ok, sms, al.ok ? bwd_vectors(block_input(a), bias, t, r, d->width) : 1);
    a.part = static_cast<float *>(workspace);
    if (d->rows > 0) {
        if (int rc = FLARE_BLOCK_TYPES(d, block_backward)(a, al.ok, bias, plan, st)) return rc;
    }
    const bool shared_gate = a.grouped && a.dg;
    if (!shared_gate && !out.d_scale && !out.dw_post && !out.db_post && !out.dw_pre && !out.db_pre) return FLARE_OK;
    BlockSums s{};
    s.part = a.part;
    s.g = a.g; s.dg = a.dg; s.ld_g = a.ld_g; s.ld_dg = a.ld_dg;
    s.scale = a.scale; s.w_post = a.w_post; s.b_post = a.b_post;
    s.d_scale = out.d_scale; s.dw_post = out.dw_post; s.db_post = out.db_post; s.dw_pre = out.dw_pre; s.db_pre = out.db_pre;
    s.groups = d->rows > 0 ? plan.groups : 0; s.chunks = plan.chunks; s.C = d->width;
    s.branch = join; s.bias = bias; s.sums = (join ? 2 : 1) * (bias ? 2 : 1);
    s.gate = a.gate; s.grouped = a.grouped;
    return d->dtype == FLARE_DTYPE_F32 ? block_sums<float>(s, st) : d->dtype == FLARE_DTYPE_BF16 ? block_sums<__nv_bfloat16>(s, st) : block_sums<__half>(s, st);
}

}  // namespace
}  // namespace flare

using namespace flare;

extern "C" {

size_t flare_block_workspace_bytes(const flare_block_desc_t *desc) {
    if (check_block(desc, true) != FLARE_OK) return 0;
    // (the norm's backward has one group of all rows whatever the descriptor's gate is, with more blocks to it than groups in all, it may be)
    return std::max(partial_bytes(desc, group_of(desc)), partial_bytes(desc, std::max<long>(desc->rows, 1)));
}

int flare_norm_forward(const flare_block_desc_t *desc, const void *x, const float *weight, const float *bias, void *h, float *stats, flare_stream_t stream) {
    if (int rc = check_block(desc, false)) return rc;
    if (desc->rows > 0 && (!x || !h)) return FLARE_ERR_INVALID_ARG;
    if (!float_params_ok({weight, bias}) || !aligned16(stats)) return FLARE_ERR_INVALID_ARG;
    BlockArgs a = common_args(desc, false);
    a.x = x; a.w_pre = weight; a.b_pre = bias; a.h = h; a.stats = reinterpret_cast<float4 *>(stats);
    return forward(desc, a, reinterpret_cast<cudaStream_t>(stream));
}

int flare_norm_backward(const flare_block_desc_t *desc, const void *x, const float *weight, const float *stats, const void *dy, const void *dh, void *dx,
                        float *dweight, float *dbias, void *workspace, size_t workspace_bytes, flare_stream_t stream) {
    if (int rc = check_block(desc, false)) return rc;
    if (desc->rows > 0 && (!x || !stats || !dh || !dx)) return FLARE_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace) || !float_params_ok({weight, dweight, dbias}) || !aligned16(stats)) return FLARE_ERR_INVALID_ARG;
    BlockArgs a = common_args(desc, false);
    a.x = x; a.w_pre = weight; a.stats = reinterpret_cast<float4 *>(const_cast<float *>(stats)); a.dy = dy; a.dh = dh; a.dx = dx;
    const BlockGrads out{nullptr, nullptr, nullptr, dweight, dbias};
    return backward(desc, false, a, out, workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}

int flare_join_forward(const flare_block_desc_t *desc, const void *x, const void *branch, const void *gate, const float *scale, const float *post_weight,
                       const float *post_bias, const float *pre_weight, const float *pre_bias, void *y, void *h, float *stats, flare_stream_t stream) {
    if (int rc = check_block(desc, true)) return rc;
    const bool pre = desc->pre_norm != FLARE_NORM_NONE, post = desc->post_norm != FLARE_NORM_NONE, gated = desc->gate != FLARE_GATE_NONE;
    if (desc->rows > 0 && (!x || !branch || !y || pre != (h != nullptr) || gated != (gate != nullptr))) return FLARE_ERR_INVALID_ARG;
    if ((!post && (post_weight || post_bias)) || (!pre && (pre_weight || pre_bias))) return FLARE_ERR_INVALID_ARG;
    if (!float_params_ok({scale, post_weight, post_bias, pre_weight, pre_bias}) || !aligned16(stats)) return FLARE_ERR_INVALID_ARG;
    BlockArgs a = common_args(desc, true);
    a.x = x; a.o = branch; a.g = gate; a.scale = scale; a.w_post = post_weight; a.b_post = post_bias; a.w_pre = pre_weight; a.b_pre = pre_bias;
    a.y = y; a.h = h; a.stats = reinterpret_cast<float4 *>(stats);
    return forward(desc, a, reinterpret_cast<cudaStream_t>(stream));
}

int flare_join_backward(const flare_block_desc_t *desc, const void *branch, const void *gate, const float *scale, const float *post_weight,
                        const float *post_bias, const void *y, const float *pre_weight, const float *stats, const void *dy, const void *dh, void *dx,
                        void *dbranch, void *dgate, float *dscale, float *dpost_weight, float *dpost_bias, float *dpre_weight, float *dpre_bias,
                        void *workspace, size_t workspace_bytes, flare_stream_t stream) {
    if (int rc = check_block(desc, true)) return rc;
    const bool pre = desc->pre_norm != FLARE_NORM_NONE, post = desc->post_norm != FLARE_NORM_NONE, gated = desc->gate != FLARE_GATE_NONE;
    if (desc->rows > 0) {
        if (!branch || !stats || !dx || !dbranch || gated != (gate != nullptr) || gated != (dgate != nullptr)) return FLARE_ERR_INVALID_ARG;
        if (pre != (dh != nullptr) || (pre && !y) || (!pre && !dy)) return FLARE_ERR_INVALID_ARG;
    }
    if ((!post && (post_weight || post_bias || dpost_weight || dpost_bias)) || (!pre && (pre_weight || dpre_weight || dpre_bias))) return FLARE_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace) || !aligned16(stats) ||
        !float_params_ok({scale, post_weight, post_bias, pre_weight, dscale, dpost_weight, dpost_bias, dpre_weight, dpre_bias}))
        return FLARE_ERR_INVALID_ARG;
    BlockArgs a = common_args(desc, true);
    a.o = branch; a.g = gate; a.scale = scale; a.w_post = post_weight; a.b_post = post_bias; a.x = y; a.w_pre = pre_weight;
    a.stats = reinterpret_cast<float4 *>(const_cast<float *>(stats)); a.dy = dy; a.dh = dh; a.dx = dx; a.d_o = dbranch; a.dg = dgate;
    const BlockGrads out{dscale, dpost_weight, dpost_bias, dpre_weight, dpre_bias};
    return backward(desc, true, a, out, workspace, workspace_bytes,
                    reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
