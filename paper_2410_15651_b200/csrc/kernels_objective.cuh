// The O(B*T) kernels of the objectives beside step 4: the sums of the policy loss with its KL term where the row kernel
// does not form them itself, and the pairs of the preference loss.
#pragma once
#include "common.cuh"
#include "kernels_generic.cuh"
#include "kernels_small.cuh"

namespace rlhf {

// Sum of one double per thread of a block of kThreads (fixed shuffle tree, then warps in index order); thread 0 gets it.
template <int kThreads>
__device__ inline double block_sum_double(double v, double* s_red /* kThreads / 32 */)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();                 // s_red is free from the previous sum
    if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = v;
    __syncthreads();
    double tot = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kThreads / 32; ++w) tot += s_red[w];
    return tot;
}

// ---------------------------------------------------------------- means of the per-token terms
// The losses of a row kernel that leaves its per-token terms in the workspace (valid tokens only): every block adds a
// contiguous range, the last block to finish adds the blocks' sums in index order.
struct RowSumArgs {
    const int* lengths;
    int B, T;
    int seq_mean;               // the terms already carry 1 / length; divide by the non-empty sequences instead of N
    const float* row_loss;
    const float* row_kl;        // optional
    float* out_lp_new;          // optional: zeroed at padded tokens here
    float* out_loss;
    float* out_kl;              // optional
    unsigned* ticket;
    double* partials;           // workspace: [kFinalMaxBlocks][2]
};

__global__ void __launch_bounds__(kFinalThreads) row_sums_kernel(RowSumArgs p)
{
    __shared__ long long s_cnt[33];
    __shared__ double s_red[kFinalThreads / 32];
    __shared__ bool s_last;
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const long long N = block_count_valid(p.lengths, p.B, p.T, s_cnt, nullptr);
    const long long D = p.seq_mean ? block_count_nonempty(p.lengths, p.B, s_cnt) : N;
    const long long total = (long long)p.B * p.T;
    const long long per_block = (total + gridDim.x - 1) / gridDim.x;
    const long long begin = per_block * blockIdx.x, end = min(total, begin + per_block);
    double sum_loss = 0.0, sum_kl = 0.0;
    for (long long i = begin + threadIdx.x; i < end; i += blockDim.x) {
        const int b = (int)(i / p.T), t = (int)(i % p.T);
        if (t < clamp_len(__ldg(p.lengths + b), p.T)) {
            sum_loss += (double)p.row_loss[i];
            if (p.row_kl) sum_kl += (double)p.row_kl[i];
        } else if (p.out_lp_new) {
            p.out_lp_new[i] = 0.f;
        }
    }
    const double bl = block_sum_double<kFinalThreads>(sum_loss, s_red);
    const double bk = block_sum_double<kFinalThreads>(sum_kl, s_red);
    if (threadIdx.x == 0) {
        p.partials[2 * blockIdx.x] = bl;
        p.partials[2 * blockIdx.x + 1] = bk;
        __threadfence();
        s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (s_last && threadIdx.x == 0) {
        __threadfence();
        double a = 0.0, c = 0.0;
        for (unsigned k = 0; k < gridDim.x; ++k) {
            a += ((volatile double*)p.partials)[2 * k];
            c += ((volatile double*)p.partials)[2 * k + 1];
        }
        *p.out_loss = D > 0 ? (float)(a / (double)D) : 0.f;
        if (p.out_kl) *p.out_kl = D > 0 ? (float)(c / (double)D) : 0.f;
        *p.ticket = 0u;
    }
}

// ---------------------------------------------------------------- pairs of the preference loss
// One block per pair (sequences i and i + B/2), half of its threads per sequence: the log ratio of each is a sum over its
// tokens, added in double precision in a fixed order; thread 0 forms the pair's loss and the factor that every token's gradient of the two
// sequences carries.  The block that finishes last adds the pairs' losses in a fixed order.
struct PairArgs {
    const float* lp;            // [B,T] log-probs of the current logits (0 at padding and at ids out of range)
    const float* lp_ref;        // [B,T] or null
    const long long* ids;
    long long ids_stride_b;
    const int* lengths;
    int B, T, V;
    int kind;                   // rlhf_preference_t
    float beta, margin, smoothing;
    int length_mean;
    float grad_scale;
    float* out_loss;
    float* out_rewards;         // [B]: beta times the log ratio
    float* seq_factor;          // workspace [B]
    double* pair_loss;          // workspace [B/2]
    unsigned* ticket;
};

constexpr int kPairThreads = 256;
constexpr int kPrefSigmoid = 0, kPrefHinge = 1, kPrefSquared = 2;

// Loss of a pair and its derivative with respect to h.  log sigma(-|h|) = -|h| - log1p(exp(-|h|)) never overflows.
__device__ inline void pair_objective(int kind, double h, double beta, double e, double& loss, double& dh)
{
    if (kind == kPrefSigmoid) {
        const double x = exp(-fabs(h));
        const double soft = log1p(x);                                  // -log sigma(|h|)
        const double lo = x / (1.0 + x), hi = 1.0 / (1.0 + x);         // sigma(-|h|), sigma(|h|)
        const double nl_pos = h >= 0.0 ? soft : soft - h;              // -log sigma(h)
        const double nl_neg = h >= 0.0 ? soft + h : soft;              // -log sigma(-h)
        loss = (1.0 - e) * nl_pos + (e == 0.0 ? 0.0 : e * nl_neg);     // (h = +inf, a rejected token that is deleted: 0)
        dh = e * (h >= 0.0 ? hi : lo) - (1.0 - e) * (h >= 0.0 ? lo : hi);
    } else if (kind == kPrefHinge) {
        loss = 1.0 - h > 0.0 ? 1.0 - h : 0.0;
        dh = h < 1.0 ? -1.0 : 0.0;
        if (!(h == h)) loss = dh = h;
    } else {
        const double d = (h - 0.5) / beta;
        loss = d * d;
        dh = 2.0 * d / beta;
    }
}

__global__ void __launch_bounds__(kPairThreads) preference_pair_kernel(PairArgs p)
{
    __shared__ double s_red[kPairThreads / 32];
    __shared__ bool s_last;
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const int half = p.B / 2;
    for (int i = blockIdx.x; i < half; i += gridDim.x) {
        const int bc = i, br = i + half;
        const int nc = clamp_len(__ldg(p.lengths + bc), p.T), nr = clamp_len(__ldg(p.lengths + br), p.T);
        // half the block per sequence: each warp leaves its sum, thread 0 adds them in warp order
        const bool rejected = threadIdx.x >= kPairThreads / 2;
        const int b = rejected ? br : bc, len = rejected ? nr : nc;
        const long long base = (long long)b * p.T;
        double s = 0.0;
        for (int t = threadIdx.x & (kPairThreads / 2 - 1); t < len; t += kPairThreads / 2) {
            const long long y = __ldg(p.ids + (long long)b * p.ids_stride_b + t);
            const float lp = p.lp[base + t], lp_ref = p.lp_ref ? __ldg(p.lp_ref + base + t) : 0.f;
            if (y >= 0 && y < p.V) s += (double)lp - (double)lp_ref;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        __syncthreads();                 // the sums of the block's previous pair have been read
        if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            double sc = 0.0, sr = 0.0;
            for (int w = 0; w < kPairThreads / 64; ++w) { sc += s_red[w]; sr += s_red[kPairThreads / 64 + w]; }
            const double wc = p.length_mean && nc > 0 ? 1.0 / nc : 1.0, wr = p.length_mean && nr > 0 ? 1.0 / nr : 1.0;
            sc *= wc;
            sr *= wr;
            const double beta = (double)p.beta;
            double loss, dh;
            pair_objective(p.kind, beta * (sc - sr) - (double)p.margin, beta, (double)p.smoothing, loss, dh);
            p.pair_loss[i] = loss;
            p.out_rewards[bc] = (float)(beta * sc);
            p.out_rewards[br] = (float)(beta * sr);
            const double f = (double)p.grad_scale * beta * dh / (double)half;
            p.seq_factor[bc] = (float)(f * wc);
            p.seq_factor[br] = (float)(-f * wr);
            if (half == 1) *p.out_loss = (float)loss;
        }
    }
    if (half == 1) return;               // a single pair: nothing to add up
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double acc = 0.0;
    for (int i = threadIdx.x; i < half; i += kPairThreads) acc += __ldcg(p.pair_loss + i);
    const double tot = block_sum_double<kPairThreads>(acc, s_red);
    if (threadIdx.x == 0) {
        *p.out_loss = (float)(tot / (double)half);
        *p.ticket = 0u;
    }
}

}  // namespace rlhf
