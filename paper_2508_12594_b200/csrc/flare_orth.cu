// Orthogonalised updates: argument checks, scales, launches.
#include "flare_host.h"
#include "flare_orth.cuh"

namespace flare {
namespace {

size_t size_of(int dtype) { return dtype == FLARE_DTYPE_F32 ? 4 : 2; }

struct OrthSizes { int S, L; long ld_x, ld_s; };
OrthSizes sizes_of(const flare_orth_desc_t *d) {
    OrthSizes z;
    z.S = std::min(d->rows, d->cols);
    z.L = std::max(d->rows, d->cols);
    z.ld_x = (z.L + 7) / 8 * 8;
    z.ld_s = (z.S + 7) / 8 * 8;
    return z;
}
bool orth_small(const OrthSizes &z) { return z.S <= 128 && orth_small_size(z.S, z.L).total <= 227 * 1024 - 512; }

// How large X, A = X X^T and B = a I + b A + c A^2 get: X0 has singular values up to 1, each step takes the largest to the quintic's largest value up
// to there.  The halves' scales put that near the top of float16's range, so that the low halves of small entries are normal numbers too.
// False where the values grow beyond what the halves are good for (a quintic that does not stay near 1).
bool orth_scales(const flare_orth_desc_t *d, OrthScales *out) {
    const double a = d->coefficients[0], b = d->coefficients[1], c = d->coefficients[2];
    double top = 1.0, x = 1.0, poly = 0.0;
    for (int step = 0; step < d->steps; ++step) {
        // largest |v q(v^2)| and |q(v^2)|, q(t) = a + b t + c t^2, for v up to `top`: at its ends and where a derivative vanishes
        const double t1 = 1.002 * top * top;
        double next = 0.0;
        auto at = [&](double t) {
            if (!(t >= 0.0) || t > t1) return;
            const double q = a + b * t + c * t * t;
            next = std::max(next, std::sqrt(t) * std::fabs(q));
            poly = std::max(poly, std::fabs(q));
        };
        at(0.0); at(t1);
        if (c != 0.0) {
            at(-b / (2.0 * c));                                            // q' = b + 2 c t
            const double root = std::sqrt(std::max(0.0, 9.0 * b * b - 20.0 * a * c));
            at((-3.0 * b + root) / (10.0 * c)); at((-3.0 * b - root) / (10.0 * c));   // (v q)' = a + 3 b t + 5 c t^2
        } else if (b != 0.0) {
            at(-a / (3.0 * b));
        }
        top = next;
        x = std::max(x, top);
        if (!(x <= 64.0) || !(poly <= 4096.0)) return false;
    }
    auto scale = [](double most) { return (float)std::exp2(std::floor(std::log2(40000.0 / most))); };
    out->x = scale(x);
    out->a = scale(x * x);
    out->b = scale(std::max(poly, 1e-3));
    out->ca = (float)a; out->cb = (float)b; out->cc = (float)c;
    return true;
}

int check_orth(const flare_orth_desc_t *d, OrthScales *scales) {
    if (d == nullptr) return FLARE_ERR_INVALID_ARG;
    if (d->count < 0 || d->rows <= 0 || d->cols <= 0 || d->steps < 1 || !(d->eps >= 0.f) || !std::isfinite(d->eps)) return FLARE_ERR_INVALID_ARG;
    for (float c : d->coefficients)
        if (!std::isfinite(c)) return FLARE_ERR_INVALID_ARG;
    if ((d->stride_row != 0 && d->stride_row < d->cols) || (d->out_stride_row != 0 && d->out_stride_row < d->cols) || d->stride_matrix < 0 || d->out_stride_matrix < 0)
        return FLARE_ERR_INVALID_ARG;
    auto type = [](int t) { return t == FLARE_DTYPE_F32 || t == FLARE_DTYPE_BF16 || t == FLARE_DTYPE_F16; };
    if (!type(d->dtype) || !type(d->weight_dtype)) return FLARE_ERR_UNSUPPORTED;
    if (d->rows > 65536 || d->cols > 65536 || d->count > 32767 || d->steps > 64 || (int64_t)d->rows * d->cols > ((int64_t)1 << 31) - 1) return FLARE_ERR_UNSUPPORTED;
    return orth_scales(d, scales) ? FLARE_OK : FLARE_ERR_UNSUPPORTED;
}

int norm_blocks(const flare_orth_desc_t *d, int sms) {
    const long each = ((long)d->rows * d->cols + kOrthNormThreads * 16 - 1) / (kOrthNormThreads * 16);
    return (int)std::max(1L, std::min(each, (8L * sms + d->count - 1) / std::max(1, d->count)));
}
// How a team does a product: blocks that share a tile's K, and of a symmetric result, whether only the upper tiles are computed.  In 64-deep steps of a
// tile (1024 cycles with all blocks at work, see below): sharing (the sums to memory, the wait, the sums from memory) costs about 6 of them, storing a
// tile's transpose 3, which a team with blocks to spare saves by computing both; each product some 9 to start and to meet.
struct TeamPlan { int ks; bool upper; double cost; };
TeamPlan team_plan(int team, long rows, long cols, bool symmetric, int K) {
    const int blocks = (K + 63) / 64;
    TeamPlan best{1, false, 0.0};
    for (int upper = 0; upper <= (symmetric ? 1 : 0); ++upper) {
        const long tiles = upper ? rows * (rows + 1) / 2 : rows * cols;
        for (int ks = 1; ks <= 8; ++ks) {
            if (ks > 1 && ks * tiles > team) break;
            const long turns = ks > 1 ? 1 : (tiles + team - 1) / team;
            const double cost = 9.0 + (double)turns * ((blocks + ks - 1) / ks + (ks > 1 ? 6 : 0) + (upper && rows > 1 ? 3 : 0));
            if (best.cost == 0.0 || cost < best.cost) best = TeamPlan{ks, upper != 0, cost};
        }
    }
    return best;
}
// Clusters of n blocks of the team kernel that the chip holds at a time (the SMs of a cluster are of one part of the chip: 33 clusters of four, 15 of
// eight, 7 of sixteen); asked for once per device, 0 = not yet.
int clusters_at_a_time(int n, int sms) {
    static std::atomic<int> known[64][17];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return n == 16 ? 7 : n == 8 ? 15 : n == 4 ? 33 : sms / n;     // (no device: for size queries)
    }
    int most = known[dev][n].load(std::memory_order_relaxed);
    if (most == 0) {
        auto *kernel = orth_team_kernel<true, float>;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = n; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)n); cfg.blockDim = kOrthThreads; cfg.dynamicSmemBytes = kOrthSmem;
        cfg.attrs = &attr; cfg.numAttrs = 1;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kOrthSmem) != cudaSuccess ||
            cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess || most < 1) {
            cudaGetLastError();
            most = -1;                                                // (cannot be placed)
        }
        known[dev][n].store(most, std::memory_order_relaxed);
    }
    return most;
}
// How a cluster of n does a product: tiles of 128 or 64 columns.  Cycles: some 4500 to start and to meet, and a turn's steps and end.
struct ClusterPlan { int width; double cost; };
ClusterPlan cluster_plan(int n, int rows, int cols, int K) {
    ClusterPlan best{0, 0.0};
    for (int width : {128, 64}) {
        const long tiles = (long)((rows + 127) / 128) * ((cols + width - 1) / width), turns = (tiles + n - 1) / n;
        const double cost = 4500.0 + (double)turns * ((K + 63) / 64 * (width == 128 ? 900.0 : 620.0) + (width == 128 ? 2600.0 : 2000.0));
        if (best.width == 0 || cost < best.cost) best = ClusterPlan{width, cost};
    }
    return best;
}
// How a problem is run.
enum { kOrthSmallPath = 0, kOrthTeamPath = 1, kOrthPairPath = 2, kOrthClusterPath = 3 };
struct OrthPlan { int path, team, teams; };
OrthPlan orth_plan(const flare_orth_desc_t *d, int sms) {
    const OrthSizes z = sizes_of(d);
    OrthPlan p{};
    if (orth_small(z)) return p;
    const int count = std::max(1, d->count);
    p.teams = std::min(count, sms);
    p.team = sms / p.teams;
    // Time of a step, in cycles: a team's as above, matrices that have to wait for a team one after the other (a tile's 64 of K are 768 cycles of matrix
    // instructions, 1024 with what all blocks load at a time); a launch per product over pairs: 1536 cycles each 64 of K and tile of four times the size,
    // and some 20000 to start, finish and follow one another.  Measured, us, teams : pairs: 256 x 256 125 : 232, 1024 x 4096 305 : 648, 2048 x 2048 454 : 685,
    // 1500 x 6000 766 : 997, four of 2048 x 2048 1889 : 1793, 2500 x 2500 1277 : 991, 3600 x 3600 2619 : 3018, 4096 x 4096 3496 : 3364, two of it 8045 : 6480.
    const double rounds = (double)((count + p.teams - 1) / p.teams);
    const long s = (z.S + 127) / 128, l = (z.L + 127) / 128, s2 = (z.S + 255) / 256, l2 = (z.L + 255) / 256;
    const double team = 1024.0 * rounds * (team_plan(p.team, s, s, true, z.L).cost + team_plan(p.team, s, s, true, z.S).cost + team_plan(p.team, s, l, false, z.S).cost);
    auto launch = [&](long tiles, int K) { return 20000.0 + (double)((tiles * count + sms / 2 - 1) / (sms / 2)) * ((K + 63) / 64) * 1536.0; };
    const double pairs = launch(s2 * (s2 + 1) / 2, z.L) + launch(s2 * (s2 + 1) / 2, z.S) + launch(s2 * l2, z.S);
    p.path = team <= pairs ? kOrthTeamPath : kOrthPairPath;
    double least = std::min(team, pairs);
    for (int n : {1, 2, 4, 8, 16}) {
        const int most = clusters_at_a_time(n, sms), clusters = std::min(count, most);
        if (most < 1) continue;
        const double cost = (double)((count + clusters - 1) / clusters) *
                            (cluster_plan(n, z.S, z.S, z.L).cost + cluster_plan(n, z.S, z.S, z.S).cost + cluster_plan(n, z.S, z.L, z.S).cost);
        if (cost < least) {
            least = cost;
            p = OrthPlan{kOrthClusterPath, n, clusters};
        }
    }
    return p;
}
struct OrthLayout { size_t counters, norm, x[2], a, b, part, total; };
OrthLayout orth_layout(const flare_orth_desc_t *d, const OrthPlan &plan, int sms) {
    const OrthSizes z = sizes_of(d);
    OrthLayout w{};
    size_t off = kHeaderBytes;
    if (plan.path != kOrthSmallPath) {
        const bool team = plan.path == kOrthTeamPath;
        const size_t n = 2 * (size_t)d->count * sizeof(__half), blocks = (size_t)plan.team * plan.teams;
        w.counters = off;
        if (team) off += align_up(sizeof(uint32_t) * (plan.teams + 3 * blocks));
        w.norm = off; off += align_up(sizeof(double) * (size_t)d->count * norm_blocks(d, sms));
        for (size_t &x : w.x) { x = off; off += align_up(n * z.S * z.ld_x); }
        w.a = off; off += align_up(n * z.S * z.ld_s);
        w.b = off; off += align_up(n * z.S * z.ld_s);
        w.part = off;
        if (team) off += blocks * 128 * 128 * sizeof(float);
    }
    w.total = off;
    return w;
}

// Halves [planes, rows, cols] of rows `ld` apart, in boxes of box_cols x box_rows: 64 columns with 128-byte swizzle, 32 with 64-byte.
int make_half_map(CUtensorMap *m, const void *base, long cols, long rows, long planes, long ld, int box_cols, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled not available");
        return FLARE_ERR_CUDA;
    }
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)rows};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled(halves) failed: %d", (int)r);
        return FLARE_ERR_CUDA;
    }
    return FLARE_OK;
}

int make_half_maps(HalfMaps *m, const void *base, long cols, long rows, long planes, long ld) {
    int rc;
    if ((rc = make_half_map(&m->load, base, cols, rows, planes, ld, 64, 64)) != FLARE_OK) return rc;
    if ((rc = make_half_map(&m->store, base, cols, rows, planes, ld, 64, 32)) != FLARE_OK) return rc;
    return make_half_map(&m->store_t, base, cols, rows, planes, ld, 32, 64);
}

template <int kKind, typename E = float>
int launch_pairs(const HalfMaps &ta, const HalfMaps &tb, const HalfMaps &out, OrthPairArgs a, int count, int sms, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    if (int rc = ensure_big_smem(orth_pair_kernel<kKind, E>, opt_in, (int)kOrthSmem)) return rc;
    OrthProduct &p = a.p;
    p.width = 256;
    p.tiles_m = (p.S + 255) / 256;
    p.tiles_n = (p.N + 255) / 256;
    p.upper = kKind == kOrthGram || kKind == kOrthPoly;
    p.per_m = 1.f / (float)p.tiles_m;
    p.tiles = p.upper ? p.tiles_n * (p.tiles_n + 1) / 2 : p.tiles_m * p.tiles_n;
    a.total = p.tiles * count;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * (unsigned)std::min(a.total, sms / 2));
    cfg.blockDim = kOrthThreads; cfg.dynamicSmemBytes = kOrthSmem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, orth_pair_kernel<kKind, E>, ta.load, tb.load, out.store, out.store_t, a));
    return FLARE_OK;
}
// Teams: a cooperative launch (its blocks wait for one another: all of them at once or none), or clusters.
template <bool kCluster, typename E>
int launch_teams(const OrthMaps &maps, const OrthTeam &p, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0}, opt_large{0};
    auto *kernel = orth_team_kernel<kCluster, E>;
    if (int rc = ensure_big_smem(kernel, opt_in, (int)kOrthSmem)) return rc;
    cudaLaunchAttribute attr[2] = {};
    int attrs = 1;
    if (kCluster) {
        int dev = 0;
        FLARE_CUDA(cudaGetDevice(&dev));
        if (!(opt_large.load(std::memory_order_acquire) >> (dev & 63) & 1)) {
            FLARE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
            opt_large.fetch_or(1ull << (dev & 63), std::memory_order_release);
        }
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = p.team; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        attrs = 2;
    } else {
        attr[0].id = cudaLaunchAttributeCooperative;
        attr[0].val.cooperative = 1;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.team * p.teams));
    cfg.blockDim = kOrthThreads; cfg.dynamicSmemBytes = kOrthSmem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = attrs;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, kernel, maps, p));
    return FLARE_OK;
}
template <typename E>
int launch_teams_as(bool cluster, const OrthMaps &maps, const OrthTeam &p, cudaStream_t st) {
    return cluster ? launch_teams<true, E>(maps, p, st) : launch_teams<false, E>(maps, p, st);
}

int run_orth(const flare_orth_desc_t *d, const OrthScales &sc, OrthOuter o, void *workspace, cudaStream_t st) {
    auto fours = [&](const void *p, long ld, long step, int type) {
        return d->cols % 4 == 0 && ld % 4 == 0 && step % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (4 * size_of(type)) == 0;
    };
    o.in_fours = fours(o.g, o.ld_g, o.step_g, o.g_type) && (!o.m || (aligned16(o.m) && aligned16(o.m_out)));
    o.out_fours = fours(o.out, o.ld_out, o.step_out, o.out_type) && (!o.w || fours(o.w, o.ld_out, o.step_out, o.out_type));
    const int sms = device_info().sms;
    const OrthSizes z = sizes_of(d);
    const OrthPlan plan = orth_plan(d, sms);
    const OrthLayout w = orth_layout(d, plan, sms);
    uint32_t *status = static_cast<uint32_t *>(workspace);
    const int words = (int)((plan.path == kOrthTeamPath ? w.norm : kHeaderBytes) / sizeof(uint32_t));
    FLARE_CUDA(launch_after(orth_clear_kernel, 1, 256, 0, st, status, words));
    if (plan.path == kOrthSmallPath) {
        OrthSmall p{};
        p.o = o; p.sc = sc; p.S = z.S; p.L = z.L; p.Mr = (z.S + 15) / 16 * 16; p.panels = (z.L + 63) / 64; p.steps = d->steps; p.status = status;
        auto launch = [&](auto kernel, std::atomic<uint64_t> &opt_in) {
            if (int rc = ensure_big_smem(kernel, opt_in, 227 * 1024 - 512)) return rc;
            FLARE_CUDA(launch_after(kernel, (unsigned)d->count, kOrthSmallThreads, orth_small_size(z.S, z.L).total, st, p));
            return (int)FLARE_OK;
        };
        static std::atomic<uint64_t> opt_narrow{0}, opt_wide{0};
        if (int rc = z.S <= 64 ? launch(orth_small_kernel<true>, opt_narrow) : launch(orth_small_kernel<false>, opt_wide)) return rc;
        return FLARE_OK;
    }
    char *ws = static_cast<char *>(workspace);
    double *norm = reinterpret_cast<double *>(ws + w.norm);
    __half *x[2] = {reinterpret_cast<__half *>(ws + w.x[0]), reinterpret_cast<__half *>(ws + w.x[1])};
    __half *A = reinterpret_cast<__half *>(ws + w.a), *B = reinterpret_cast<__half *>(ws + w.b);
    const int parts = norm_blocks(d, sms);
    FLARE_CUDA(launch_after(orth_norm_kernel, dim3(parts, d->count), kOrthNormThreads, 0, st, o, norm));
    FLARE_CUDA(launch_after(orth_split_kernel, dim3(parts, d->count), 256, 0, st, o, norm, parts, x[0], z.ld_x, sc.x));
    const long planes = 2L * d->count;
    HalfMaps tx[2], tA, tB;
    int rc;
    for (int i = 0; i < 2; ++i)
        if ((rc = make_half_maps(&tx[i], x[i], z.L, z.S, planes, z.ld_x)) != FLARE_OK) return rc;
    if ((rc = make_half_maps(&tA, A, z.S, z.S, planes, z.ld_s)) != FLARE_OK) return rc;
    if ((rc = make_half_maps(&tB, B, z.S, z.S, planes, z.ld_s)) != FLARE_OK) return rc;
    if (plan.path == kOrthTeamPath || plan.path == kOrthClusterPath) {
        const bool cluster = plan.path == kOrthClusterPath;
        OrthTeam p{};
        p.o = o;
        for (int kind = 0; kind < 4; ++kind) {
            OrthProduct &q = p.product[kind];
            const bool symmetric = kind == kOrthGram || kind == kOrthPoly;
            q.a = A; q.ld_a = z.ld_s; q.S = z.S; q.N = symmetric ? z.S : z.L; q.K = kind == kOrthGram ? z.L : z.S;
            q.width = cluster ? cluster_plan(plan.team, q.S, q.N, q.K).width : 128;
            q.tiles_m = (q.S + 127) / 128; q.tiles_n = (q.N + q.width - 1) / q.width;
            const TeamPlan how = cluster ? TeamPlan{1, false, 0.0} : team_plan(plan.team, q.tiles_m, q.tiles_n, symmetric, q.K);
            q.upper = how.upper; p.ks[kind] = how.ks;
            q.tiles = q.upper ? q.tiles_n * (q.tiles_n + 1) / 2 : q.tiles_m * q.tiles_n;
            q.per_m = 1.f / (float)q.tiles_m;
            q.f = kind == kOrthGram ? sc.a / (sc.x * sc.x) : kind == kOrthPoly ? sc.cc * sc.b / (sc.a * sc.a) : kind == kOrthApply ? 1.f / sc.b : 1.f / (sc.b * sc.x);
            q.fa = sc.cb * sc.b / sc.a; q.fi = sc.ca * sc.b;
        }
        const OrthMaps maps{{tx[0], tx[1], tA, tB}};
        p.mem[0] = x[0]; p.mem[1] = x[1]; p.mem[2] = A; p.mem[3] = B;
        p.part = reinterpret_cast<float *>(ws + w.part);
        p.counters = reinterpret_cast<uint32_t *>(ws + w.counters); p.status = status;
        p.ld_x = z.ld_x; p.ld_s = z.ld_s; p.S = z.S; p.L = z.L; p.count = d->count; p.steps = d->steps; p.team = plan.team; p.teams = plan.teams;
        return o.out_type == FLARE_DTYPE_F32    ? launch_teams_as<float>(cluster, maps, p, st)
               : o.out_type == FLARE_DTYPE_BF16 ? launch_teams_as<__nv_bfloat16>(cluster, maps, p, st)
                                                : launch_teams_as<__half>(cluster, maps, p, st);
    }
    for (int step = 0; step < d->steps; ++step) {
        const int cur = step & 1;
        OrthPairArgs a{};
        OrthProduct &p = a.p;
        a.status = status; p.S = z.S; p.N = z.S;
        p.K = z.L; p.f = sc.a / (sc.x * sc.x);
        if ((rc = launch_pairs<kOrthGram>(tx[cur], tx[cur], tA, a, d->count, sms, st)) != FLARE_OK) return rc;
        p.a = A; p.ld_a = z.ld_s; p.K = z.S;
        p.f = sc.cc * sc.b / (sc.a * sc.a); p.fa = sc.cb * sc.b / sc.a; p.fi = sc.ca * sc.b;
        if ((rc = launch_pairs<kOrthPoly>(tA, tA, tB, a, d->count, sms, st)) != FLARE_OK) return rc;
        p.N = z.L;
        if (step + 1 < d->steps) {
            p.f = 1.f / sc.b;
            if ((rc = launch_pairs<kOrthApply>(tB, tx[cur], tx[1 - cur], a, d->count, sms, st)) != FLARE_OK) return rc;
        } else {
            a.o = o;
            p.f = 1.f / (sc.b * sc.x);
            auto last = o.out_type == FLARE_DTYPE_F32    ? launch_pairs<kOrthLast, float>
                        : o.out_type == FLARE_DTYPE_BF16 ? launch_pairs<kOrthLast, __nv_bfloat16>
                                                         : launch_pairs<kOrthLast, __half>;
            if ((rc = last(tB, tx[cur], tx[1 - cur], a, d->count, sms, st)) != FLARE_OK) return rc;
        }
    }
    return FLARE_OK;
}

bool natural(const void *p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

int need_device() {
    const DeviceView di = device_info();
    if (di.checked == -2) {
        snprintf(g_cuda_error, sizeof(g_cuda_error), "no CUDA device");
        return FLARE_ERR_CUDA;
    }
    return di.checked == 1 ? FLARE_OK : FLARE_ERR_ARCH;
}

// No matrices: the header says that no wait gave up, whatever the workspace held.
int clear_header(void *workspace, cudaStream_t st) {
    FLARE_CUDA(launch_after(orth_clear_kernel, 1, 256, 0, st, static_cast<uint32_t *>(workspace), (int)(kHeaderBytes / sizeof(uint32_t))));
    return FLARE_OK;
}

OrthOuter outer_of(const flare_orth_desc_t *d) {
    OrthOuter o{};
    o.rows = d->rows; o.cols = d->cols; o.g_type = d->dtype; o.eps = d->eps; o.tall = d->rows > d->cols;
    o.ld_g = d->stride_row ? d->stride_row : d->cols;
    o.step_g = d->stride_matrix ? d->stride_matrix : o.ld_g * d->rows;
    return o;
}

}  // namespace
}  // namespace flare

using namespace flare;

extern "C" {

size_t flare_orthogonalize_workspace_bytes(const flare_orth_desc_t *desc) {
    OrthScales sc;
    if (check_orth(desc, &sc) != FLARE_OK) return 0;
    return orth_layout(desc, orth_plan(desc, device_info().sms), device_info().sms).total;
}

int flare_orthogonalize_plan(const flare_orth_desc_t *desc, int32_t plan[3]) {
    OrthScales sc;
    if (int rc = check_orth(desc, &sc)) return rc;
    if (!plan) return FLARE_ERR_INVALID_ARG;
    const OrthPlan p = orth_plan(desc, device_info().sms);
    const bool groups = p.path == kOrthTeamPath || p.path == kOrthClusterPath;
    plan[0] = p.path; plan[1] = groups ? p.team : 0; plan[2] = groups ? p.teams : 0;
    return FLARE_OK;
}

int flare_orthogonalize(const flare_orth_desc_t *desc, const void *G, void *O, void *workspace, size_t workspace_bytes, flare_stream_t stream) {
    OrthScales sc;
    if (int rc = check_orth(desc, &sc)) return rc;
    const size_t e = size_of(desc->dtype);
    if (!workspace || !aligned16(workspace) || (desc->count > 0 && (!G || !O)) || !natural(G, e) || !natural(O, e)) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    if (workspace_bytes < orth_layout(desc, orth_plan(desc, device_info().sms), device_info().sms).total) return FLARE_ERR_WORKSPACE_TOO_SMALL;
    if (desc->count == 0) return clear_header(workspace, reinterpret_cast<cudaStream_t>(stream));
    OrthOuter o = outer_of(desc);
    o.g = G; o.out = O; o.out_type = desc->dtype;
    o.ld_out = desc->out_stride_row ? desc->out_stride_row : desc->cols;
    o.step_out = desc->out_stride_matrix ? desc->out_stride_matrix : o.ld_out * desc->rows;
    return run_orth(desc, sc, o, workspace, reinterpret_cast<cudaStream_t>(stream));
}

int flare_muon_update(const flare_orth_desc_t *desc, const flare_muon_t *rule, const void *w, const float *m, const void *g, void *w_out, float *m_out,
                      void *workspace, size_t workspace_bytes, flare_stream_t stream) {
    OrthScales sc;
    if (int rc = check_orth(desc, &sc)) return rc;
    if (!rule || !std::isfinite(rule->lr) || !std::isfinite(rule->momentum) || !std::isfinite(rule->weight_decay) || !std::isfinite(rule->update_scale))
        return FLARE_ERR_INVALID_ARG;
    const size_t e = size_of(desc->weight_dtype);
    if (!workspace || !aligned16(workspace) || (desc->count > 0 && (!w || !m || !g || !w_out || !m_out))) return FLARE_ERR_INVALID_ARG;
    if (!natural(w, e) || !natural(w_out, e) || !natural(m, 4) || !natural(m_out, 4) || !natural(g, size_of(desc->dtype))) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    if (workspace_bytes < orth_layout(desc, orth_plan(desc, device_info().sms), device_info().sms).total) return FLARE_ERR_WORKSPACE_TOO_SMALL;
    if (desc->count == 0) return clear_header(workspace, reinterpret_cast<cudaStream_t>(stream));
    OrthOuter o = outer_of(desc);
    o.g = g; o.w = w; o.out = w_out; o.out_type = desc->weight_dtype; o.m = m; o.m_out = m_out;
    o.ld_out = desc->cols; o.step_out = (long)desc->cols * desc->rows;
    o.nesterov = rule->nesterov != 0; o.momentum = rule->momentum;
    o.keep = 1.f - rule->lr * rule->weight_decay; o.rate = rule->lr * rule->update_scale;
    return run_orth(desc, sc, o, workspace, reinterpret_cast<cudaStream_t>(stream));
}

int flare_selftest_team(void *workspace, int32_t gone, uint64_t budget_ns, flare_stream_t stream) {
    if (!workspace || !aligned16(workspace) || gone < 0 || gone > 2) return FLARE_ERR_INVALID_ARG;
    if (int rc = need_device()) return rc;
    budget_ns = std::min<uint64_t>(std::max<uint64_t>(budget_ns, 1000), 100000000ull);   // never more than a tenth of a second
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    uint32_t *words = static_cast<uint32_t *>(workspace);
    FLARE_CUDA(cudaMemsetAsync(workspace, 0, 2 * kHeaderBytes, st));
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeCooperative;
    attr.val.cooperative = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2); cfg.blockDim = kOrthThreads; cfg.stream = st;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, selftest_team_kernel, words, words + kHeaderBytes / 4, words + kHeaderBytes / 4 + 1, (int)gone, budget_ns));
    return FLARE_OK;
}

}  // extern "C"
