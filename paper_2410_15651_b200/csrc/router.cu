// Entry points of the router's balance loss: argument checks and launches.
#include <algorithm>

#include "common.cuh"
#include "host.cuh"
#include "kernels_router.cuh"

namespace {

using namespace rlhf;

struct RouterPlan {
    long long groups = 0, n_chunks = 0, n_partials = 0;
    int cluster = 1;
};

// Chunks of at least 32 tokens, enough of them to fill the device.  Groups of more than 48 chunks are counted by clusters, so that
// a block of the second launch has at most 48 partial counts per expert to add.
RouterPlan plan_router(int L, int B, int T, bool per_sequence)
{
    RouterPlan p;
    p.groups = (long long)L * (per_sequence ? B : 1);
    const long long rows = per_sequence ? T : (long long)B * T;
    const long long most = std::min<long long>(kRouterMaxChunks, std::max<long long>(1, rows / 32));
    p.n_chunks = std::min(most, std::max<long long>(1, kRouterTargetBlocks / p.groups));
    if (p.n_chunks > 48) {
        p.cluster = kRouterCluster;
        p.n_chunks = p.n_chunks / kRouterCluster * kRouterCluster;
    }
    p.n_partials = p.n_chunks / p.cluster;
    return p;
}

// The losses' parts (16 bytes a block), then the partial counts.
size_t router_bytes(const RouterPlan& p, int E)
{
    return kRowLossOffset + 16 * (size_t)(p.groups * p.n_chunks) + 4 * (size_t)(p.groups * p.n_partials) * (size_t)E;
}

bool router_shape_ok(int L, int B, int T, int E)
{
    return L > 0 && B > 0 && T > 0 && E > 0 && E <= kRouterMaxExperts && (long long)B * T <= kMaxTokens &&
           (long long)L * ((long long)B * T) <= kMaxTokens;
}

template <int kType, int NV, int G>
int launch_router_as(const RouterArgs& a, int grid, cudaStream_t s)
{
    if (int e = keep_max_carveout(router_count_kernel<kType, NV, G>)) return e;
    RLHF_CUDA(launch_kernel_cluster(router_count_kernel<kType, NV, G>, grid, kRouterThreads, 0, a.cluster, s, a));
    if (int e = launch_check("router_count_kernel")) return e;
    if (int e = keep_max_carveout(router_loss_kernel<kType, NV, G>)) return e;
    RLHF_CUDA(launch_kernel(router_loss_kernel<kType, NV, G>, grid, kRouterThreads, 0, s, a));
    return launch_check("router_loss_kernel");
}

// Lanes of a token and vectors of eight logits per lane.  16-bit logits: two vectors (24 x 16 x 1024 tokens of 128 experts, K = 8:
// 148 us, with one vector and twice the lanes 176 us, in the same number of blocks), fp32 one, and more where a warp would not do.
template <int kType>
int launch_router(RouterArgs& a, int grid, cudaStream_t s)
{
    if (a.E > 512) return launch_router_as<kType, 4, 32>(a, grid, s);
    if (a.E > 256) return launch_router_as<kType, 2, 32>(a, grid, s);
    if (a.E <= 8) return launch_router_as<kType, 1, 1>(a, grid, s);
    constexpr int NV = kType == RLHF_F32 ? 1 : 2;
    switch (router_lanes(a.E, NV)) {
        case 1: return launch_router_as<kType, NV, 1>(a, grid, s);
        case 2: return launch_router_as<kType, NV, 2>(a, grid, s);
        case 4: return launch_router_as<kType, NV, 4>(a, grid, s);
        case 8: return launch_router_as<kType, NV, 8>(a, grid, s);
        case 16: return launch_router_as<kType, NV, 16>(a, grid, s);
        default: return launch_router_as<kType, 1, 32>(a, grid, s);
    }
}

}  // namespace

extern "C" {

size_t rlhf_router_workspace_bytes(int L, int B, int T, int E)
{
    if (!router_shape_ok(L, B, T, E)) return 0;
    const size_t n = std::max(router_bytes(plan_router(L, B, T, false), E), router_bytes(plan_router(L, B, T, true), E));
    return (n + 255) & ~(size_t)255;
}

int rlhf_router_loss_fwd_bwd(const void* logits, int logits_dtype, long long stride_l, long long stride_b, long long stride_t,
                             const int* expert_ids, long long ids_stride_l, long long ids_stride_b, long long ids_stride_t,
                             const int* lengths, int L, int B, int T, int E, int K, int scoring, int scope,
                             float balance_coef, float z_coef, float grad_scale, float* out_loss, int* out_counts, int* out_ids,
                             void* out_dlogits, long long dl_stride_l, long long dl_stride_b, long long dl_stride_t,
                             void* workspace, size_t workspace_bytes, void* stream)
{
    if (!logits || !lengths || !out_loss || !out_counts || !out_dlogits) return RLHF_ERR_NULL;
    if (logits_dtype != RLHF_BF16 && logits_dtype != RLHF_F16 && logits_dtype != RLHF_F32) return RLHF_ERR_SCALAR;
    if (!router_shape_ok(L, B, T, E) || K <= 0 || K > E) return RLHF_ERR_SHAPE;
    if ((scoring != RLHF_ROUTER_SOFTMAX && scoring != RLHF_ROUTER_SIGMOID) || (scope != RLHF_ROUTER_BATCH && scope != RLHF_ROUTER_SEQUENCE) ||
        !std::isfinite(balance_coef) || !std::isfinite(z_coef) || !std::isfinite(grad_scale) ||
        (scoring != RLHF_ROUTER_SOFTMAX && z_coef != 0.f))
        return RLHF_ERR_SCALAR;
    if (stride_l < 0 || stride_b < 0 || stride_t < 0 || dl_stride_l < 0 || dl_stride_b < 0 || dl_stride_t < 0 ||
        ids_stride_l < 0 || ids_stride_b < 0 || ids_stride_t < 0)
        return RLHF_ERR_STRIDE;
    // the gradient's rows do not overlap: layer, sequence and token axes in this order, or sequence, token, layer and the like
    // (an axis of one position has no stride)
    {
        long long st[3] = {dl_stride_l, dl_stride_b, dl_stride_t};
        int n[3] = {L, B, T};
        long long span = E;
        for (int done = 0; done < 3; ++done) {
            int k = -1;
            for (int i = 0; i < 3; ++i)
                if (n[i] > 1 && (k < 0 || st[i] < st[k])) k = i;
            if (k < 0) break;
            if (st[k] < span) return RLHF_ERR_STRIDE;
            span += (long long)(n[k] - 1) * st[k];
            n[k] = 1;
        }
    }
    if (out_dlogits == logits && ((L > 1 && dl_stride_l != stride_l) || (B > 1 && dl_stride_b != stride_b) || (T > 1 && dl_stride_t != stride_t)))
        return RLHF_ERR_STRIDE;
    const size_t size = logits_dtype == RLHF_F32 ? 4 : 2;
    if (!aligned(logits, size) || !aligned(out_dlogits, size) || !aligned(expert_ids, 4) || !aligned(lengths, 4) ||
        !aligned(out_loss, 4) || !aligned(out_counts, 4) || !aligned(out_ids, 4))
        return RLHF_ERR_ALIGN;
    const RouterPlan p = plan_router(L, B, T, scope == RLHF_ROUTER_SEQUENCE);
    if (int e = check_workspace(workspace, workspace_bytes, router_bytes(p, E))) return e;

    char* ws = (char*)workspace;
    RouterArgs a{};
    a.logits = logits;
    a.stride_l = stride_l; a.stride_b = stride_b; a.stride_t = stride_t;
    a.lengths = lengths;
    a.L = L; a.B = B; a.T = T; a.E = E; a.K = K;
    a.ids_in = expert_ids;
    a.ids_stride_l = ids_stride_l; a.ids_stride_b = ids_stride_b; a.ids_stride_t = ids_stride_t;
    a.scoring = scoring == RLHF_ROUTER_SOFTMAX ? kRouterSoftmax : kRouterSigmoid;
    a.per_sequence = scope == RLHF_ROUTER_SEQUENCE;
    a.balance_coef = balance_coef;
    a.z_coef = z_coef;
    a.grad_scale = grad_scale;
    a.out_loss = out_loss;
    a.out_counts = out_counts;
    a.out_ids = expert_ids ? nullptr : out_ids;
    a.dlogits = out_dlogits;
    a.dl_stride_l = dl_stride_l; a.dl_stride_b = dl_stride_b; a.dl_stride_t = dl_stride_t;
    a.status = (unsigned*)ws;
    a.ticket = (unsigned*)(ws + 4);
    a.partial_loss = (double*)(ws + kRowLossOffset);
    a.partial_counts = (int*)(ws + kRowLossOffset + 16 * (size_t)(p.groups * p.n_chunks));
    a.groups = (int)p.groups;
    a.n_chunks = (int)p.n_chunks;
    a.n_partials = (int)p.n_partials;
    a.cluster = p.cluster;
    const long long per = (long long)(16 / size);
    auto vec = [&](const void* base, long long sl, long long sb, long long st) {
        return E % 8 == 0 && aligned(base, 16) && (L == 1 || sl % per == 0) && (B == 1 || sb % per == 0) && (T == 1 || st % per == 0);
    };
    a.vec_in = vec(logits, stride_l, stride_b, stride_t);
    a.vec_out = vec(out_dlogits, dl_stride_l, dl_stride_b, dl_stride_t);
    a.flat_in = a.per_sequence || B == 1 || T == 1 || stride_b == (long long)T * stride_t;
    a.flat_out = a.per_sequence || B == 1 || T == 1 || dl_stride_b == (long long)T * dl_stride_t;
    // (rows of single tokens follow each other at the sequences' stride)
    if (T == 1 && !a.per_sequence) {
        a.stride_t = stride_b;
        a.dl_stride_t = dl_stride_b;
    }
    // division by T: ceil(2^(32 + shift) / T), shift the bits of T - 1
    while ((1ll << a.t_shift) < T) ++a.t_shift;
    a.t_shift = a.t_shift > 0 ? a.t_shift - 1 : 0;
    a.t_magic = (unsigned)(((1ull << (32 + a.t_shift)) + (unsigned)T - 1) / (unsigned)T);
    const int grid = (int)(p.groups * p.n_chunks);
    cudaStream_t s = (cudaStream_t)stream;
    if (logits_dtype == RLHF_BF16) return launch_router<0>(a, grid, s);
    if (logits_dtype == RLHF_F16) return launch_router<1>(a, grid, s);
    return launch_router<2>(a, grid, s);
}

}  // extern "C"
