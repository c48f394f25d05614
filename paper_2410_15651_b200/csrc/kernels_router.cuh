// Balance loss of an expert router, with the experts' counts and the gradient.
//
// For a token with router logits z over E experts, p = softmax(z) or sigmoid(z) / sum sigmoid(z), and K chosen experts; for a
// group of n tokens (all of a layer's, or one sequence's of it) with c_e choices of expert e,
//     balance = (1/n) sum_tokens sum_e f_e p_e,   f_e = E c_e / (K n),        zloss = (1/N) sum_tokens lse(z)^2.
// The counts are constants of the gradient, so a token's share needs nothing of the others' probabilities:
//     d balance / d z_j = (1/n) s_j p_j (f_j - sum_e f_e p_e),   s_j = 1 (softmax) or 1 - sigmoid(z_j),
// and the loss is the sum of the same dot products.  With f_e - 1 in place of f_e (both dots have sum p = 1) nothing is lost
// where the experts are nearly balanced.
//
// Two launches: counts, then losses and gradient.  A token is held by G = 1 .. 32 lanes with 8 (16, 32 above 256, 512
// experts) consecutive entries each.  Both are bound by HBM in the large and by their two launches in the small; the second
// walks the tokens backwards, so that what the first read last comes from L2.
#pragma once
#include "common.cuh"

namespace rlhf {

constexpr int kRouterThreads = 256;
constexpr int kRouterMaxExperts = 1024;
constexpr int kRouterMaxChunks = 256;        // chunks of a group (partial counts: one per kRouterCluster of them)
constexpr int kRouterCluster = 8;
constexpr int kRouterTargetBlocks = 1184;

enum : int { kRouterSoftmax = 0, kRouterSigmoid = 1 };

struct RouterArgs {
    const void* logits;
    long long stride_l, stride_b, stride_t;
    const int* lengths;
    int L, B, T, E, K;
    const int* ids_in;                       // chosen experts, or null: the K largest logits
    long long ids_stride_l, ids_stride_b, ids_stride_t;
    int scoring, per_sequence;
    float balance_coef, z_coef, grad_scale;
    float* out_loss;                         // [L,2]
    int* out_counts;                         // [L,E], or [L,B,E] per sequence
    int* out_ids;                            // [L,B,T,K], or null
    void* dlogits;
    long long dl_stride_l, dl_stride_b, dl_stride_t;
    unsigned* status;
    unsigned* ticket;
    int* partial_counts;                     // [groups][n_partials][E]
    double* partial_loss;                    // [blocks][2]
    int groups, n_chunks, n_partials, chunk_rows;
    int cluster;                             // blocks of the counting kernel that share a partial count
    int lanes, per_lane;                     // G, and entries of a lane
    int vec_in, vec_out;                     // rows can be moved in 16-byte pieces
};

// The element types: 16-bit as elsewhere, and fp32.
template <int kType> struct RouterEl;        // rlhf_dtype_t
template <> struct RouterEl<0> { using T = uint16_t; static __device__ __forceinline__ float get(uint16_t v) { return El<false>::widen(v); } };
template <> struct RouterEl<1> { using T = uint16_t; static __device__ __forceinline__ float get(uint16_t v) { return El<true>::widen(v); } };
template <> struct RouterEl<2> { using T = float; static __device__ __forceinline__ float get(float v) { return v; } };

// Which tokens a block has: rows [r0, r1) of group g.  A row is (b, t).
struct RouterItem {
    int g, l, r0, r1, b0;                    // b0: the sequence of a per-sequence group
};

__device__ __forceinline__ RouterItem router_item(const RouterArgs& a, int block)
{
    RouterItem it;
    it.g = block / a.n_chunks;
    const int chunk = block % a.n_chunks, rows = a.per_sequence ? a.T : a.B * a.T;
    it.l = a.per_sequence ? it.g / a.B : it.g;
    it.b0 = a.per_sequence ? it.g % a.B : 0;
    it.r0 = (int)min((long long)chunk * a.chunk_rows, (long long)rows);
    it.r1 = (int)min((long long)it.r0 + a.chunk_rows, (long long)rows);
    return it;
}

__device__ __forceinline__ void router_row(const RouterArgs& a, const RouterItem& it, int r, int& b, int& t)
{
    if (a.per_sequence) { b = it.b0; t = r; }
    else { b = r / a.T; t = r - b * a.T; }
}

// Entries e0 .. e0 + 8 NV - 1 of a row; `missing` past E.
template <int kType, int NV>
__device__ __forceinline__ void router_load(const typename RouterEl<kType>::T* row, int e0, int E, bool vec, float missing,
                                            float (&z)[8 * NV])
{
    using Ty = typename RouterEl<kType>::T;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = e0 + 8 * v;
        float* o = z + 8 * v;
        if (vec && e < E) {                  // E is a multiple of 8 then
            if constexpr (sizeof(Ty) == 2) {
                const uint4 q = __ldg((const uint4*)(row + e));
                const float2 p0 = El<kType == 1>::unpack2(q.x), p1 = El<kType == 1>::unpack2(q.y), p2 = El<kType == 1>::unpack2(q.z),
                             p3 = El<kType == 1>::unpack2(q.w);
                o[0] = p0.x; o[1] = p0.y; o[2] = p1.x; o[3] = p1.y; o[4] = p2.x; o[5] = p2.y; o[6] = p3.x; o[7] = p3.y;
            } else {
                const float4 q = __ldg((const float4*)(row + e)), w = __ldg((const float4*)(row + e) + 1);
                o[0] = q.x; o[1] = q.y; o[2] = q.z; o[3] = q.w; o[4] = w.x; o[5] = w.y; o[6] = w.z; o[7] = w.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = e + j < E ? RouterEl<kType>::get(row[e + j]) : missing;
        }
    }
}

template <int kType, int NV>
__device__ __forceinline__ void router_store(typename RouterEl<kType>::T* row, int e0, int E, bool vec, const float (&d)[8 * NV])
{
    using Ty = typename RouterEl<kType>::T;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = e0 + 8 * v;
        const float* x = d + 8 * v;
        if constexpr (sizeof(Ty) == 2) {
            const uint4 w = make_uint4(El<kType == 1>::pack2(x[0], x[1]), El<kType == 1>::pack2(x[2], x[3]),
                                       El<kType == 1>::pack2(x[4], x[5]), El<kType == 1>::pack2(x[6], x[7]));
            if (vec && e < E) {
                __stcs((uint4*)(row + e), w);
            } else {
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e + j < E) row[e + j] = (uint16_t)(ww[j >> 1] >> (16 * (j & 1)));
            }
        } else {
            if (vec && e < E) {
                __stcs((float4*)(row + e), make_float4(x[0], x[1], x[2], x[3]));
                __stcs((float4*)(row + e) + 1, make_float4(x[4], x[5], x[6], x[7]));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e + j < E) row[e + j] = x[j];
            }
        }
    }
}

// Unsigned order of floats; -0 and 0 are equal, a number that does not exist (0) is below -inf.
__device__ __forceinline__ uint32_t router_key(float z)
{
    const uint32_t u = __float_as_uint(z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// ---------------------------------------------------------------- counts
template <int kType, int NV>
__global__ void __launch_bounds__(kRouterThreads) router_count_kernel(const __grid_constant__ RouterArgs a)
{
    using Ty = typename RouterEl<kType>::T;
    __shared__ int s_count[kRouterMaxExperts];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int e = tid; e < a.E; e += kRouterThreads) s_count[e] = 0;
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    if (blockIdx.x == 0) {                   // what is wrong with the lengths is said once
        for (int b = tid; b < a.B; b += kRouterThreads) {
            const int n = __ldg(a.lengths + b);
            if (n < 0 || n > a.T) atomicOr(a.status, kErrLengthRange);
        }
    }
    __syncthreads();
    const RouterItem it = router_item(a, (int)blockIdx.x);

    if (a.ids_in) {
        bool bad = false;
        const int* base = a.ids_in + (long long)it.l * a.ids_stride_l;
        for (int r = it.r0 + tid; r < it.r1; r += kRouterThreads) {
            int b, t;
            router_row(a, it, r, b, t);
            if (t >= __ldg(a.lengths + b)) continue;
            const int* ids = base + (long long)b * a.ids_stride_b + (long long)t * a.ids_stride_t;
            for (int k = 0; k < a.K; ++k) {
                const int e = __ldg(ids + k);
                if (e >= 0 && e < a.E) atomicAdd(s_count + e, 1);
                else if (e != -1) bad = true;
            }
        }
        if (bad) atomicOr(a.status, kErrIdRange);
    } else {
        const int G = a.lanes, sub = lane & (G - 1), per_warp = 32 / G;
        const int e0 = sub * 8 * NV;
        const uint32_t group = (G == 32 ? 0xffffffffu : ((1u << G) - 1u)) << (lane & ~(G - 1));
        const int step = kRouterThreads / 32 * per_warp;
        // (every lane of a warp makes every turn: the shuffles want them all)
        for (int r = it.r0 + warp * per_warp; r < it.r1; r += step) {
            const int mine = r + lane / G;
            int b = 0, t = 0;
            bool row = mine < it.r1, valid = false;
            if (row) {
                router_row(a, it, mine, b, t);
                valid = t < __ldg(a.lengths + b);
            }
            uint32_t key[8 * NV];
            if (valid) {
                float z[8 * NV];
                router_load<kType, NV>((const Ty*)a.logits + (long long)it.l * a.stride_l + (long long)b * a.stride_b + (long long)t * a.stride_t,
                                       e0, a.E, a.vec_in, 0.f, z);
#pragma unroll
                for (int j = 0; j < 8 * NV; ++j) key[j] = e0 + j < a.E ? router_key(z[j]) : 0u;
            } else {
#pragma unroll
                for (int j = 0; j < 8 * NV; ++j) key[j] = 0u;
            }
            int* out = a.out_ids ? a.out_ids + (((long long)it.l * a.B + b) * a.T + t) * a.K : nullptr;
            for (int k = 0; k < a.K; ++k) {
                uint32_t top = key[0];
                int at = 0;
#pragma unroll
                for (int j = 1; j < 8 * NV; ++j)
                    if (key[j] > top) { top = key[j]; at = j; }
                uint32_t best = top;
                for (int o = G >> 1; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                const uint32_t who = __ballot_sync(0xffffffffu, top == best) & group;
                if (lane == __ffs(who) - 1) {            // the lowest expert of those that are equal
                    const int e = min(e0 + at, a.E - 1);
                    if (valid) atomicAdd(s_count + e, 1);
                    if (out && row) out[k] = valid ? e : 0;
#pragma unroll
                    for (int j = 0; j < 8 * NV; ++j)
                        if (j == at) key[j] = 0u;
                }
            }
        }
    }
    __syncthreads();
    const int C = a.cluster;
    int* out = a.partial_counts + (long long)(blockIdx.x / (unsigned)C) * a.E;
    if (C == 1) {
        for (int e = tid; e < a.E; e += kRouterThreads) out[e] = s_count[e];
        return;
    }
    // one partial count for the cluster: a block sums its share of the experts over all blocks
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const int rank = (int)(blockIdx.x % (unsigned)C);
    for (int e = rank * kRouterThreads + tid; e < a.E; e += C * kRouterThreads) {
        int n = 0;
        for (int c = 0; c < C; ++c) {
            uint32_t at;
            int v;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                         : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(s_count + e)), "r"(c));
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at));
            n += v;
        }
        out[e] = n;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------- losses and gradient
template <int kType, int NV>
__global__ void __launch_bounds__(kRouterThreads) router_loss_kernel(const __grid_constant__ RouterArgs a)
{
    using Ty = typename RouterEl<kType>::T;
    __shared__ float s_f[kRouterMaxExperts];             // f_e - 1
    __shared__ long long s_n[33];
    __shared__ double s_sum[2][kRouterThreads / 32];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const int blocks = (int)gridDim.x, block = blocks - 1 - (int)blockIdx.x;
    const RouterItem it = router_item(a, block);
    const long long N = block_count_valid(a.lengths, a.B, a.T, s_n, nullptr);
    const long long filled = a.per_sequence ? block_count_nonempty(a.lengths, a.B, s_n) : 1;
    const long long n = a.per_sequence ? clamp_len(__ldg(a.lengths + it.b0), a.T) : N;     // tokens of the group
    const double per = n > 0 ? (double)a.E / ((double)a.K * (double)n) : 0.0;
    for (int e = tid; e < a.E; e += kRouterThreads) {
        const int* part = a.partial_counts + (long long)it.g * a.n_partials * a.E + e;
        int c = 0;
#pragma unroll 8
        for (int i = 0; i < a.n_partials; ++i) c += part[(long long)i * a.E];
        s_f[e] = (float)((double)c * per - 1.0);
        if (block % a.n_chunks == 0) a.out_counts[(long long)it.g * a.E + e] = c;
    }
    __syncthreads();

    const double wd = n > 0 ? 1.0 / ((double)n * (double)filled) : 0.0, zd = N > 0 ? 1.0 / (double)N : 0.0;
    const float wb = (float)((double)a.grad_scale * a.balance_coef * wd), wz = (float)((double)a.grad_scale * a.z_coef * 2.0 * zd);
    const int G = a.lanes, sub = lane & (G - 1), per_warp = 32 / G;
    const int e0 = sub * 8 * NV;
    const int step = kRouterThreads / 32 * per_warp;
    double sum_b = 0.0, sum_z = 0.0;
    for (int r = it.r0 + warp * per_warp; r < it.r1; r += step) {
        const int mine = r + lane / G;
        int b = 0, t = 0;
        const bool row = mine < it.r1;
        bool valid = false;
        if (row) {
            router_row(a, it, mine, b, t);
            valid = t < __ldg(a.lengths + b);
        }
        float p[8 * NV], slope[8 * NV];
        if (valid)
            router_load<kType, NV>((const Ty*)a.logits + (long long)it.l * a.stride_l + (long long)b * a.stride_b + (long long)t * a.stride_t,
                                   e0, a.E, a.vec_in, -INFINITY, p);
        else {
#pragma unroll
            for (int j = 0; j < 8 * NV; ++j) p[j] = -INFINITY;
        }
        float m = 0.f, total = 0.f, dot = 0.f;
        if (a.scoring == kRouterSoftmax) {
            m = p[0];
#pragma unroll
            for (int j = 1; j < 8 * NV; ++j) m = fmaxf(m, p[j]);
            for (int o = G >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (m == -INFINITY) m = 0.f;                 // (no token, or one that may not choose: p = 0)
#pragma unroll
            for (int j = 0; j < 8 * NV; ++j) p[j] = ex2((p[j] - m) * kLog2e);
        } else {
#pragma unroll
            for (int j = 0; j < 8 * NV; ++j) {
                const float e = ex2(-fabsf(p[j]) * kLog2e), inv = 1.f / (1.f + e);
                slope[j] = p[j] >= 0.f ? e * inv : inv;
                p[j] = p[j] >= 0.f ? inv : e * inv;
            }
        }
#pragma unroll
        for (int j = 0; j < 8 * NV; ++j) {
            total += p[j];
            if (e0 + j < a.E) dot = fmaf(p[j], s_f[e0 + j], dot);
        }
        for (int o = G >> 1; o > 0; o >>= 1) {
            total += __shfl_xor_sync(0xffffffffu, total, o);
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        const float inv = total > 0.f ? 1.f / total : (total == 0.f ? 0.f : total);
        dot *= inv;
        float lse = 0.f;
        if (a.scoring == kRouterSoftmax && total > 0.f) lse = m + logf(total);
        if (row) {
            const float gz = a.z_coef != 0.f ? wz * lse : 0.f;
            float d[8 * NV];
#pragma unroll
            for (int j = 0; j < 8 * NV; ++j) {
                const float f = e0 + j < a.E ? s_f[e0 + j] : 0.f;
                float v = wb * (f - dot);
                if (a.scoring == kRouterSigmoid) v *= slope[j];
                d[j] = valid ? (p[j] * inv) * (v + gz) : 0.f;
            }
            router_store<kType, NV>((Ty*)a.dlogits + (long long)it.l * a.dl_stride_l + (long long)b * a.dl_stride_b + (long long)t * a.dl_stride_t,
                                    e0, a.E, a.vec_out, d);
        }
        if (valid && sub == 0) {
            if (total != 0.f) sum_b += 1.0 + (double)dot;    // (0: a token that may choose no expert)
            if (a.z_coef != 0.f) sum_z += (double)lse * (double)lse;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum_b += __shfl_xor_sync(0xffffffffu, sum_b, o);
        sum_z += __shfl_xor_sync(0xffffffffu, sum_z, o);
    }
    if (lane == 0) { s_sum[0][warp] = sum_b; s_sum[1][warp] = sum_z; }
    __syncthreads();
    if (tid == 0) {
        double x = 0.0, y = 0.0;
        for (int w = 0; w < kRouterThreads / 32; ++w) { x += s_sum[0][w]; y += s_sum[1][w]; }
        a.partial_loss[2 * (long long)block] = x * wd;
        a.partial_loss[2 * (long long)block + 1] = y * zd;
        __threadfence();
        s_last = atomicAdd(a.ticket, 1u) == (unsigned)blocks - 1u;
    }
    __syncthreads();
    if (!s_last) return;
    // the last block adds each layer's parts, in an order of their own
    __threadfence();
    const int per_layer = blocks / a.L;
    for (int l = warp; l < a.L; l += kRouterThreads / 32) {
        double x = 0.0, y = 0.0;
        for (int i = lane; i < per_layer; i += 32) {
            const double2 v = __ldcg((const double2*)(a.partial_loss + 2 * ((long long)l * per_layer + i)));
            x += v.x;
            y += v.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            x += __shfl_xor_sync(0xffffffffu, x, o);
            y += __shfl_xor_sync(0xffffffffu, y, o);
        }
        if (lane == 0) {
            a.out_loss[2 * l] = (float)x;
            a.out_loss[2 * l + 1] = (float)y;
        }
    }
    if (tid == 0) *a.ticket = 0u;
}

}  // namespace rlhf
