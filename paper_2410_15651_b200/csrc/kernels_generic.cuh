// Row kernels for any layout: element-wise global loads and stores, no alignment requirement.
// They serve rows that the 16-byte fast path cannot take (odd V, odd strides, odd base address).
// One block walks the valid rows k = blockIdx.x, blockIdx.x + gridDim.x, ...; each row is read
// from global memory (twice in the loss kernel: once for the partition sum, once for the gradient,
// the second read coming from L2).
#pragma once
#include "common.cuh"

namespace rlhf {

struct RowArgs {
    const uint16_t* logits;     // bf16 bit patterns
    long long stride_b, stride_t;
    const long long* ids;
    long long ids_stride_b;
    const int* lengths;
    int B, T, V;
    unsigned* status;           // workspace word 0
    unsigned long long wait_limit_ns;   // bound of every wait on a shared-memory barrier (row kernels with a producer)
    // step 1
    float* out_lp;
    // step 4
    const float* lp_old;
    const float* adv;
    float clip_eps, grad_scale;
    uint16_t* dlogits;
    long long dl_stride_b, dl_stride_t;
    float* row_loss;            // workspace: per-token policy loss term
    float* out_lp_new;          // optional
    // step 4, finalisation fused into the row kernel (fused != 0): value loss, dvalues and both scalar losses
    int fused;
    const float* values_new;
    const float* values_old;
    const float* returns;
    float value_clip;
    float* out_dvalues;
    float* out_loss_pg;
    float* out_loss_vf;
    unsigned* ticket;           // workspace word 1, zero between calls
    double* partials;           // workspace: [gridDim.x][2] block partial sums (policy, value)
    // which objective the row belongs to (kObjPpo: step 4), and what the others take beside lp_old and adv
    int objective;
    const float* lp_ref;        // kObjPolicyKl: reference log-probs, or null (no KL term)
    long long adv_stride_b, adv_stride_t;   // kObjPolicyKl: adv[b*adv_stride_b + t*adv_stride_t]
    float ratio_lo, ratio_hi;   // kObjPolicyKl: bounds of the clipped ratio
    float kl_coef;
    int seq_mean;               // kObjPolicyKl: a token weighs 1 / (non-empty sequences * its sequence's length)
    float* row_kl;              // kObjPolicyKl: workspace, per-token KL term
    const float* seq_factor;    // kObjPreference: d(grad_scale * loss) / d(log-prob of any token of sequence b)
};

// ---------------------------------------------------------------- objectives of a row with one generated token
constexpr int kObjPpo = 0, kObjPolicyKl = 1, kObjPreference = 2, kObjDistill = 3;

// What a row's objective needs beside its log-prob; loaded ahead of the row.
struct RowScalars {
    float lp_old, adv;          // kObjPreference: adv is the sequence's factor
    float lp_ref, w;            // kObjPolicyKl
};

__device__ __forceinline__ RowScalars load_row_scalars(const RowArgs& p, int b, int t, long long flat)
{
    RowScalars s{0.f, 0.f, 0.f, 1.f};
    if (p.objective == kObjPpo) {
        s.lp_old = __ldg(p.lp_old + flat);
        s.adv = __ldg(p.adv + flat);
    } else if (p.objective == kObjPolicyKl) {
        s.lp_old = __ldg(p.lp_old + flat);
        s.adv = __ldg(p.adv + (long long)b * p.adv_stride_b + (long long)t * p.adv_stride_t);
        if (p.lp_ref) s.lp_ref = __ldg(p.lp_ref + flat);
        if (p.seq_mean) s.w = 1.f / (float)clamp_len(__ldg(p.lengths + b), p.T);
    } else {
        s.adv = __ldg(p.seq_factor + b);
    }
    return s;
}

// exp(d) - 1 - d without cancellation: the Taylor series where it is short (|d| <= 1/2: the first term left out is
// below 2^-25 of the sum), else the difference (inf at d = inf, a token that the row deletes).
__device__ __forceinline__ float exp_excess(float d)
{
    if (d > 100.f) return expm1f(d);                  // inf
    if (fabsf(d) > 0.5f) return expm1f(d) - d;
    float s = 1.f / 3628800.f;
    s = fmaf(s, d, 1.f / 362880.f);
    s = fmaf(s, d, 1.f / 40320.f);
    s = fmaf(s, d, 1.f / 5040.f);
    s = fmaf(s, d, 1.f / 720.f);
    s = fmaf(s, d, 1.f / 120.f);
    s = fmaf(s, d, 1.f / 24.f);
    s = fmaf(s, d, 1.f / 6.f);
    s = fmaf(s, d, 0.5f);
    return s * d * d;
}

// The row's log-prob from its partition sum, for the objectives beside step 4, rounded once: the terms are combined in double
// precision, so that what remains is the sum's own error (row_finish forms lse first, whose last place is that of the largest
// logit).  For one thread of a row.
__device__ __forceinline__ float lp_relative(const Acc& a, float zy)
{
    return (float)(0.6931471805599453 * ((double)zy * (double)kLog2e - (double)a.M - log2_split(a.s + a.ey)));
}

// A token of kObjPolicyKl.  A whole block waits for the gradient once per row, so that it forms it by a short chain on the
// hardware's ex2 and lg2 (kFast; relative error about 2^-22, as in row_finish_fast).  1 - exp(d) loses its relative accuracy at
// small d: its absolute error of about 2^-22 is that of lp, and so of d, itself (half a step of fp32 from 4 to 8 is 2^-22), also where
// it is the whole gradient (a clipped token, an advantage of 0).  The loss terms are formed by one thread, without the shortcuts.
struct PolicyTerm {
    float lp, unclipped, clipped;
    bool free;                  // the unclipped branch is active
};
template <bool kFast>
__device__ __forceinline__ PolicyTerm policy_term(const RowArgs& p, const RowScalars& s, const Acc& tot, float zy)
{
    PolicyTerm q;
    q.lp = kFast ? kLn2 * (fmaf(zy, kLog2e, -tot.M) - lg2(tot.s + tot.ey)) : lp_relative(tot, zy);
    const float rho = kFast ? ex2((q.lp - s.lp_old) * kLog2e) : expf(q.lp - s.lp_old);
    // (an advantage of 0, a group of equal scores, has no policy part at a ratio beyond fp32 either: not 0 * inf)
    q.unclipped = -s.adv * (s.adv == 0.f && rho > 1.f ? 1.f : rho);
    q.clipped = -s.adv * fminf(fmaxf(rho, p.ratio_lo), p.ratio_hi);
    q.free = !(q.unclipped < q.clipped);                              // NaN stays in
    return q;
}
// g = d(grad_scale * total loss) / d(log-prob).  `scale` is grad_scale over the number of tokens (or of non-empty sequences).
__device__ __forceinline__ float policy_gradient(const RowArgs& p, const RowScalars& s, const PolicyTerm& q, float scale)
{
    const float d_pg = q.free ? q.unclipped : 0.f;
    // (kl_coef = 0 reports the KL without training on it: 0 * inf, where the reference is 89 nats above or more, is not formed)
    const float d_kl = p.lp_ref && p.kl_coef != 0.f ? p.kl_coef * (1.f - ex2((s.lp_ref - q.lp) * kLog2e)) : 0.f;
    return scale * s.w * (d_pg + d_kl);
}
// The token's terms in the two losses.
__device__ __forceinline__ void policy_loss_terms(const RowArgs& p, const RowScalars& s, const PolicyTerm& q, float& loss, float& kl)
{
    loss = s.w * (q.free ? q.unclipped : q.clipped);
    kl = p.lp_ref ? s.w * exp_excess(s.lp_ref - q.lp) : 0.f;
}

// Loss terms of one token and its g.  lp is replaced by the value the objective is formed with.
template <bool kFast>
__device__ __forceinline__ void row_objective(const RowArgs& p, const RowScalars& s, const Acc& tot, float zy, float& lp,
                                              float scale, float& loss, float& kl, float& g)
{
    kl = 0.f;
    if (p.objective == kObjPpo) {
        ppo_token<kFast>(lp, s.lp_old, s.adv, p.clip_eps, scale, loss, g);
    } else if (p.objective == kObjPolicyKl) {
        const PolicyTerm q = policy_term<kFast>(p, s, tot, zy);
        lp = q.lp;
        g = policy_gradient(p, s, q, scale);
        policy_loss_terms(p, s, q, loss, kl);
    } else {
        loss = 0.f;
        g = s.adv;
    }
}

constexpr int kGenericThreads = 256;

// Block-wide merge of per-thread partial sums; every thread returns the total.
__device__ inline Acc block_merge(Acc a, Acc* smem /* >= 32 */)
{
    a = acc_warp_reduce(a);
    int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5;
    __syncthreads();                 // smem free from the previous row
    if (lane == 0) smem[warp] = a;
    __syncthreads();
    Acc r = smem[0];
    for (int w = 1; w < nw; ++w) r = acc_merge(r, smem[w]);
    return r;
}

// kF16: logits and gradient are IEEE binary16 instead of bf16.
template <bool kLoss, bool kF16 = false>
__global__ void __launch_bounds__(kGenericThreads) row_generic_kernel(RowArgs p)
{
    __shared__ Acc s_acc[32];
    __shared__ long long s_cnt[33];
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const long long N = block_count_valid(p.lengths, p.B, p.T, s_cnt, blockIdx.x == 0 ? p.status : nullptr);
    const long long D = kLoss && p.seq_mean ? block_count_nonempty(p.lengths, p.B, s_cnt) : N;
    const float scale_over_N = N > 0 ? p.grad_scale / (float)D : 0.f;

    Cursor cur{0, 0};
    for (long long k = blockIdx.x; k < N; k += gridDim.x) {
        int b, t;
        if (!cursor_seek_valid(cur, k, p.lengths, p.B, p.T, b, t)) break;
        const long long flat = (long long)b * p.T + t;
        long long y = __ldg(p.ids + (long long)b * p.ids_stride_b + t);
        const bool bad_id = (y < 0 || y >= p.V);
        if (bad_id) { y = 0; if (threadIdx.x == 0) atomicOr(p.status, kErrIdRange); }
        const uint16_t* row = p.logits + (long long)b * p.stride_b + (long long)t * p.stride_t;

        // every thread reads z_y before the block barrier, i.e. before any in-place write of this row
        const float zy = El<kF16>::widen(row[y]);
        Acc a = acc_empty();
        const bool apart = kLoss && p.objective != kObjPpo;
        if (apart)
            for (int v = threadIdx.x; v < p.V; v += blockDim.x) acc_add<true>(a, El<kF16>::widen(row[v]), v == (int)y);
        else
            for (int v = threadIdx.x; v < p.V; v += blockDim.x) acc_add(a, El<kF16>::widen(row[v]), v == (int)y);
        a = block_merge(a, s_acc);
        RowResult r = row_finish(a, zy);

        if (!kLoss) {
            if (threadIdx.x == 0) p.out_lp[flat] = bad_id ? 0.f : r.lp;
            continue;
        }
        float loss = 0.f, kl = 0.f, g = 0.f;
        if (!bad_id) row_objective<false>(p, load_row_scalars(p, b, t, flat), a, zy, r.lp, scale_over_N, loss, kl, g);
        if (threadIdx.x == 0) {
            if (p.row_loss) p.row_loss[flat] = loss;
            if (p.row_kl) p.row_kl[flat] = kl;
            if (p.out_lp_new) p.out_lp_new[flat] = bad_id ? 0.f : r.lp;
        }
        uint16_t* drow = p.dlogits + (long long)b * p.dl_stride_b + (long long)t * p.dl_stride_t;
        if (g == 0.f) {
            for (int v = threadIdx.x; v < p.V; v += blockDim.x) drow[v] = 0;
        } else {
            // |g| * p_v = 2^(x_v - lse2 + log2|g|); the sign is applied to the packed result
            // (as one constant in step 4; beside it as -M and the rest, which keeps its last places in rows far from 0)
            const float c2 = apart ? -a.M : log2f(fabsf(g)) - r.lse2;
            const float rest = apart ? log2f(fabsf(g)) - log2f(a.s + a.ey) : 0.f;
            const uint16_t sign = g > 0.f ? 0x8000u : 0u;
            for (int v = threadIdx.x; v < p.V; v += blockDim.x) {
                float z = El<kF16>::widen(row[v]);                    // read before the in-place write
                float d = ex2(fmaf(z, kLog2e, c2) + rest);
                uint16_t h = (uint16_t)(El<kF16>::pack2(d, 0.f) & 0xffffu) ^ sign;
                if (v == (int)y) h = (uint16_t)(El<kF16>::pack2(g * r.one_m_py, 0.f) & 0xffffu);
                drow[v] = h;
            }
        }
    }

    if (kLoss) {
        // zero rows for padded tokens
        const long long n_pad = (long long)p.B * p.T - N;
        Cursor pc{0, 0};
        for (long long k = blockIdx.x; k < n_pad; k += gridDim.x) {
            int b, t;
            if (!cursor_seek_padded(pc, k, p.lengths, p.B, p.T, b, t)) break;
            uint16_t* drow = p.dlogits + (long long)b * p.dl_stride_b + (long long)t * p.dl_stride_t;
            for (int v = threadIdx.x; v < p.V; v += blockDim.x) drow[v] = 0;
        }
    } else {
        // log-prob 0 at padded tokens
        const long long total = (long long)p.B * p.T;
        for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total;
             i += (long long)gridDim.x * blockDim.x) {
            int b = (int)(i / p.T), t = (int)(i % p.T);
            if (t >= clamp_len(__ldg(p.lengths + b), p.T)) p.out_lp[i] = 0.f;
        }
    }
}

}  // namespace rlhf
