// Launches of the kernels around a block (flare_block.cuh) for one pair of types: T of the branch, the gate and the normalised rows,
// R of the residual stream.  Instantiated by flare_block_{bf16,bf16_f32,f16,f16_f32,f32}.cu.
#pragma once

#include "flare_block.cuh"
#include "flare_host.h"

namespace flare {

// Threads of a block: 512 for rows that 256 with their groups of eight columns do not hold, else 256.  What a row has beyond that goes to further blocks
// of a cluster.
constexpr int kBlockMaxWidth = 16384;
// Blocks per group of rows: together about as many as fill the chip once.
struct BlockPlan {
    int tpr, threads, cluster;
    long groups;
    int chunks;                                             // blocks per group
};
inline BlockPlan block_plan(long rows, long group, int C, bool aligned, int sms, int vectors) {    // vectors: groups of eight columns a thread owns
    BlockPlan p;
    p.threads = C > 2048 * vectors ? 512 : 256;
    p.tpr = aligned ? 4 : 32;                               // (rows off 16-byte boundaries: a warp copies its 256 columns together, its lanes own every 32nd)
    while (p.tpr * 8 * vectors < C && p.tpr < p.threads) p.tpr *= 2;
    p.cluster = 1;
    while (p.cluster * p.threads * 8 * vectors < C) p.cluster *= 2;
    const long turn = p.threads / p.tpr, fit = (p.threads == 512 ? 1 : 2) * (long)sms / p.cluster;
    p.groups = rows / group;
    p.chunks = (int)std::max(1L, std::min(fit / std::max(1L, p.groups), (group + turn - 1) / turn));
    return p;
}

// Groups of eight columns a thread owns in the backward.  Two where there is no branch: its sums leave the registers for them, and what a row costs
// beside its elements counts half (32768 rows of 1024, rms: 41 us instead of 51).  With a branch and a 16-bit stream two where a row of one group
// a thread would take a block of 512 (8192 rows of 4096, rms, gate: 107 us instead of 113), with biases, whose sums do not fit, where it would take a
// cluster (4096 rows of 8192: rms, gate 116 instead of 199; layer, biases 158 instead of 202); narrower rows lose by it (65536 rows of 512: 105
// instead of 90), and with a float32 stream, or a gate and biases, the slots would not fit into shared memory.
constexpr bool bwd_wide(int in, bool bias, size_t size, size_t res) { return size == 2 && in != kAlone && res == 2 && !(in == kGated && bias); }
constexpr int bwd_vectors(int in, bool bias, size_t size, size_t res, int C) {
    return size == 2 && (in == kAlone || (bwd_wide(in, bias, size, res) && C > (bias ? 4096 : 2048))) ? 2 : 1;
}
// Weights of theirs that are kept in shared memory.
constexpr int bwd_weights(int in, bool bias, int vectors) { return vectors == 1 ? 0 : in == kAlone ? (bias ? 1 : 0) : 2; }
inline int block_input(const BlockArgs &a) { return a.o == nullptr ? kAlone : !a.gate ? kPlain : a.grouped ? kShared : kGated; }

template <typename T, typename R> int block_forward(const BlockArgs &a, bool aligned, int sms, cudaStream_t st);
template <typename T, typename R> int block_backward(const BlockArgs &a, bool aligned, bool bias, const BlockPlan &plan, cudaStream_t st);
template <typename T> int block_sums(const BlockSums &s, cudaStream_t st);

#ifdef FLARE_BLOCK_INSTANTIATE
template <typename Kernel>
int block_launch(Kernel kernel, std::atomic<uint64_t> &opt_in, BlockArgs a, const BlockPlan &p, size_t smem, cudaStream_t st) {
    a.tpr = p.tpr; a.chunks = p.chunks; a.cluster = p.cluster;
    if (int rc = ensure_big_smem(kernel, opt_in, 224 * 1024)) return rc;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = p.cluster; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.groups * p.chunks), p.cluster);
    cfg.blockDim = p.threads; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = p.cluster > 1 ? 2 : 1;
    FLARE_CUDA(cudaLaunchKernelEx(&cfg, kernel, a));
    return FLARE_OK;
}

template <typename T, typename R, bool kAligned, int kIn, bool kBias, int kV, int kThreads>
int block_forward_as(const BlockArgs &a, const BlockPlan &p, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    constexpr int stages = stages_for(fwd_pieces<T, R, kIn>() * kV), bias_slots = kBias && kV == 2 ? 4 * kV : 0;
    return block_launch(block_forward_kernel<T, R, kAligned, kIn, kBias, kV, kThreads>, opt_in, a, p,
                        (size_t)stages * fwd_stage<T, R, kAligned, kIn, kV, kThreads>() + bias_slots * 16 * kThreads, st);
}
template <typename T, typename R, int kIn, bool kBias, int kV>
int block_forward_aligned(const BlockArgs &a, const BlockPlan &p, cudaStream_t st) {
    return p.threads == 512 ? block_forward_as<T, R, true, kIn, kBias, kV, 512>(a, p, st) : block_forward_as<T, R, true, kIn, kBias, kV, 256>(a, p, st);
}
template <typename T, typename R, int kIn>
int block_forward_of(const BlockArgs &a, bool aligned, int sms, cudaStream_t st) {
    constexpr int kV = sizeof(T) == 2 ? 2 : 1;              // (float32: its loads fill shared memory with one group of columns a thread)
    const BlockPlan p = block_plan(a.rows, a.group, a.C, aligned, sms, aligned ? kV : 1);
    // (rows off 16-byte boundaries: always the form with biases, here and in the backward)
    if (!aligned) return p.threads == 512 ? block_forward_as<T, R, false, kIn, true, 1, 512>(a, p, st) : block_forward_as<T, R, false, kIn, true, 1, 256>(a, p, st);
    return a.b_post || a.b_pre ? block_forward_aligned<T, R, kIn, true, kV>(a, p, st) : block_forward_aligned<T, R, kIn, false, kV>(a, p, st);
}
template <typename T, typename R>
int block_forward(const BlockArgs &a, bool aligned, int sms, cudaStream_t st) {
    switch (block_input(a)) {
        case kAlone: return block_forward_of<T, R, kAlone>(a, aligned, sms, st);
        case kPlain: return block_forward_of<T, R, kPlain>(a, aligned, sms, st);
        case kGated: return block_forward_of<T, R, kGated>(a, aligned, sms, st);
        default: return block_forward_of<T, R, kShared>(a, aligned, sms, st);
    }
}

template <typename T, typename R, bool kAligned, int kIn, bool kBias, int kV, int kThreads, bool kOnce>
int block_backward_in(const BlockArgs &a, const BlockPlan &p, cudaStream_t st) {
    static std::atomic<uint64_t> opt_in{0};
    constexpr int stages = stages_for(bwd_pieces<T, R, kIn>() * kV), sums = bwd_sums<kIn != kAlone, kBias>();
    const size_t meet = (size_t)(kThreads / std::max(p.tpr, 32)) * sums * 8 * kV * p.tpr * sizeof(float);
    const size_t smem = std::max((size_t)stages * bwd_stage<T, R, kAligned, kIn, kV, kThreads>() + bwd_weights(kIn, kBias, kV) * 2 * kV * 16 * kThreads, meet);
    return block_launch(block_backward_kernel<T, R, kAligned, kIn, kBias, kOnce, kV, kThreads>, opt_in, a, p, smem, st);
}
// The sums of both norms in one round where a round is long (a cluster's: 4096 rows of 8192 with a float32 stream, rms, 176 us instead of 225) or
// there are four of them (layer norms over 8192 rows of 4096: 112 instead of 123).  Two of rms norms in a block take less than what one round
// adds to the arithmetic (65536 rows of 512: 90 instead of 96), and two groups of columns leave no registers for it.
template <typename T, typename R, bool kAligned, int kIn, bool kBias, int kV, int kThreads>
int block_backward_as(const BlockArgs &a, const BlockPlan &p, cudaStream_t st) {
    if constexpr (kIn != kAlone && kV == 1)
        if (p.tpr > 32 && a.has_pre && a.has_post && (p.cluster > 1 || a.layer_pre || a.layer_post))
            return block_backward_in<T, R, kAligned, kIn, kBias, kV, kThreads, true>(a, p, st);
    return block_backward_in<T, R, kAligned, kIn, kBias, kV, kThreads, false>(a, p, st);
}
template <typename T, typename R, int kIn, bool kBias>
int block_backward_aligned(const BlockArgs &a, const BlockPlan &p, cudaStream_t st) {
    constexpr int kV = bwd_vectors(kIn, kBias, sizeof(T), sizeof(R), 1);
    if constexpr (bwd_wide(kIn, kBias, sizeof(T), sizeof(R))) {
        if (bwd_vectors(kIn, kBias, sizeof(T), sizeof(R), a.C) == 2) {
            if constexpr (!kBias)
                if (p.threads == 256) return block_backward_as<T, R, true, kIn, kBias, 2, 256>(a, p, st);
            return block_backward_as<T, R, true, kIn, kBias, 2, 512>(a, p, st);
        }
    }
    return p.threads == 512 ? block_backward_as<T, R, true, kIn, kBias, kV, 512>(a, p, st) : block_backward_as<T, R, true, kIn, kBias, kV, 256>(a, p, st);
}
template <typename T, typename R, int kIn>
int block_backward_of(const BlockArgs &a, bool aligned, bool bias, const BlockPlan &p, cudaStream_t st) {
    if (!aligned) return p.threads == 512 ? block_backward_as<T, R, false, kIn, true, 1, 512>(a, p, st) : block_backward_as<T, R, false, kIn, true, 1, 256>(a, p, st);
    return bias ? block_backward_aligned<T, R, kIn, true>(a, p, st) : block_backward_aligned<T, R, kIn, false>(a, p, st);
}
template <typename T, typename R>
int block_backward(const BlockArgs &a, bool aligned, bool bias, const BlockPlan &p, cudaStream_t st) {
    switch (block_input(a)) {
        case kAlone: return block_backward_of<T, R, kAlone>(a, aligned, bias, p, st);
        case kPlain: return block_backward_of<T, R, kPlain>(a, aligned, bias, p, st);
        case kGated: return block_backward_of<T, R, kGated>(a, aligned, bias, p, st);
        default: return block_backward_of<T, R, kShared>(a, aligned, bias, p, st);
    }
}
template <typename T>
int block_sums(const BlockSums &a, cudaStream_t st) {
    FLARE_CUDA(launch_after(block_sums_kernel<T>, dim3((a.C + kSumLanes - 1) / kSumLanes, a.branch ? 2 : 1), kSumLanes * kSumSlices, 0, st, a));
    return FLARE_OK;
}
#endif

}  // namespace flare
