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
    int groups, n_chunks, n_partials;
    int cluster;                             // blocks of the counting kernel that share a partial count
    int vec_in, vec_out;                     // rows can be moved in 16-byte pieces
    int flat_in, flat_out;                   // all rows of a layer follow each other at stride_t
    unsigned t_magic;                        // for divisions by T
    int t_shift;
};

// The element types: 16-bit as elsewhere, and fp32.
template <int kType> struct RouterEl;        // rlhf_dtype_t
template <> struct RouterEl<0> { using T = uint16_t; static __device__ __forceinline__ float get(uint16_t v) { return El<false>::widen(v); } };
template <> struct RouterEl<1> { using T = uint16_t; static __device__ __forceinline__ float get(uint16_t v) { return El<true>::widen(v); } };
template <> struct RouterEl<2> { using T = float; static __device__ __forceinline__ float get(float v) { return v; } };

// Which tokens a block has: of group g the rows (a row is (b, t)) in turns of `turn` rows, every n_chunks-th of them, so that
// padding is shared out.
struct RouterItem {
    int g, l, chunk, rows, b0;               // b0: the sequence of a per-sequence group
};

__device__ __forceinline__ RouterItem router_item(const RouterArgs& a, int block)
{
    RouterItem it;
    it.g = block / a.n_chunks;
    it.chunk = block % a.n_chunks;
    it.rows = a.per_sequence ? a.T : a.B * a.T;
    it.l = a.per_sequence ? it.g / a.B : it.g;
    it.b0 = a.per_sequence ? it.g % a.B : 0;
    return it;
}

// Row r of an item, its sequence and token, and whether it is a token of the sequence.
struct RouterRow {
    int r, b, t;
    bool row, valid;
};
__device__ __forceinline__ RouterRow router_row(const RouterArgs& a, const RouterItem& it, int r)
{
    RouterRow w{r, it.b0, r, r < it.rows, false};
    if (!w.row) return w;
    if (!a.per_sequence) {
        // r / T by a product with 2^(32 + shift) / T, rounded up: T <= 2^(shift + 1), so that it is exact for r < 2^31
        w.b = a.T == 1 ? r : (int)(__umulhi((unsigned)r, a.t_magic) >> a.t_shift);
        w.t = r - w.b * a.T;
    }
    w.valid = w.t < __ldg(a.lengths + w.b);
    return w;
}
// Its offset in a tensor; `flat`: its rows follow each other at stride_t.
__device__ __forceinline__ long long router_at(const RouterRow& w, bool flat, long long stride_b, long long stride_t)
{
    return flat ? (long long)w.r * stride_t : (long long)w.b * stride_b + (long long)w.t * stride_t;
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

// Lanes of a token.
__host__ __device__ constexpr int router_lanes(int E, int nv)
{
    int g = 1;
    while (g * 8 * nv < E) g *= 2;
    return g;
}

// Two 16-bit logits in the order of unsigned numbers, -0 as 0.
template <bool kF16>
__device__ __forceinline__ uint32_t router_order2(uint32_t w)
{
    if (kF16) asm("add.rn.f16x2 %0, %0, %1;" : "+r"(w) : "r"(0u));
    else asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(w) : "r"(0u));
    const uint32_t negative = ((w >> 15) & 0x00010001u) * 0xffffu;
    return w ^ (negative | 0x80008000u);
}

// ---------------------------------------------------------------- counts
template <int kType, int NV, int G>
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
        const int choices = kRouterThreads * a.K;        // of a turn, a choice per thread
        for (int r0 = it.chunk * kRouterThreads; r0 < it.rows; r0 += a.n_chunks * kRouterThreads)
            for (int i = tid; i < choices; i += kRouterThreads) {
                const int row = i / a.K, k = i - row * a.K;
                const RouterRow w = router_row(a, it, r0 + row);
                if (!w.valid) continue;
                const int e = __ldg(base + (long long)w.b * a.ids_stride_b + (long long)w.t * a.ids_stride_t + k);
                if (e >= 0 && e < a.E) atomicAdd(s_count + e, 1);
                else if (e != -1) bad = true;
            }
        if (bad) atomicOr(a.status, kErrIdRange);
    } else {
        // 16-bit logits of one vector per lane: a key orders logit and expert at once (the higher logit, then the lower expert).  A
        // lane sorts its eight, and every turn takes the largest head.  Else a turn looks for the largest of all.
        constexpr bool kSorted = sizeof(Ty) == 2 && NV == 1;
        constexpr int kPerWarp = 32 / G, kTurn = kRouterThreads / 32 * kPerWarp;
        const int sub = lane & (G - 1), e0 = sub * 8 * NV;
        const uint32_t group = (G == 32 ? 0xffffffffu : ((1u << (G & 31)) - 1u)) << (lane & ~(G - 1));
        const Ty* const base = (const Ty*)a.logits + (long long)it.l * a.stride_l + (a.per_sequence && a.flat_in ? it.b0 * a.stride_b : 0);
        int* const ids_base = a.out_ids + ((long long)it.l * a.B + it.b0) * a.T * a.K;
        const int mine = warp * kPerWarp + lane / G;
        const int step = a.n_chunks * kTurn;
        int r = it.chunk * kTurn;
        RouterRow w = router_row(a, it, r + mine);
        float z[8 * NV];
        uint4 q = make_uint4(0, 0, 0, 0);                // kSorted and vec_in: the lane's logits as they are
        auto load = [&]() {
            if (!w.valid) return;
            const Ty* row = base + router_at(w, a.flat_in, a.stride_b, a.stride_t);
            if (kSorted && a.vec_in) {
                if (e0 < a.E) q = __ldg((const uint4*)(row + e0));
            } else {
                router_load<kType, NV>(row, e0, a.E, a.vec_in, 0.f, z);
            }
        };
        load();
        // (every lane of a warp makes every turn: the shuffles want them all)
        for (; r < it.rows; r += step) {
            const bool row = w.row, valid = w.valid;
            int* const out = a.out_ids && row ? ids_base + (long long)w.r * a.K : nullptr;
            uint32_t key[8 * NV];
            if (kSorted && a.vec_in) {
                if (valid && e0 < a.E) {
                    const uint32_t x[4] = {router_order2<kType == 1>(q.x), router_order2<kType == 1>(q.y), router_order2<kType == 1>(q.z),
                                           router_order2<kType == 1>(q.w)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        key[2 * j] = (x[j] << 16) + (0xffffu - (uint32_t)(e0 + 2 * j));
                        key[2 * j + 1] = (x[j] & 0xffff0000u) | (0xffffu - (uint32_t)(e0 + 2 * j + 1));
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) key[j] = 0u;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8 * NV; ++j) {
                    key[j] = valid && e0 + j < a.E ? router_key(z[j]) : 0u;
                    // (the low 13 bits of a 16-bit logit's key say nothing, and there are at most 256 experts; the top bits of the low
                    // half are the logit's in this form and 1 in the other)
                    if (kSorted && key[j]) key[j] = (max(key[j], 0x100u) & 0xffffff00u) | (0xffu - (uint32_t)(e0 + j));
                }
            }
            w = router_row(a, it, r + step + mine);
            load();                                      // in flight meanwhile
            if (__ballot_sync(0xffffffffu, valid) == 0u) {             // (rows of padding)
                if (out)
                    for (int k = sub; k < a.K; k += G) out[k] = 0;
                continue;
            }
            if constexpr (kSorted) {
                auto order = [&](int x, int y) {         // the larger first
                    const uint32_t hi = max(key[x], key[y]), lo = min(key[x], key[y]);
                    key[x] = hi;
                    key[y] = lo;
                };
                // Batcher's odd-even merge of eight
                order(0, 1); order(2, 3); order(4, 5); order(6, 7);
                order(0, 2); order(1, 3); order(4, 6); order(5, 7);
                order(1, 2); order(5, 6);
                order(0, 4); order(1, 5); order(2, 6); order(3, 7);
                order(2, 4); order(3, 5);
                order(1, 2); order(3, 4); order(5, 6);
                auto top = [&]() {
                    uint32_t best = key[0];
#pragma unroll
                    for (int o = G / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    return best;
                };
                if (G >= 8 && a.K <= 8) {                // lane k of a token keeps its k-th choice
                    uint32_t got = 0u;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (k >= a.K) break;
                        const uint32_t best = top();
                        const bool won = key[0] == best;
                        if (sub == k) got = best;
#pragma unroll
                        for (int j = 0; j < 7 - k; ++j) key[j] = won ? key[j + 1] : key[j];
                    }
                    if (sub < a.K) {
                        const int e = got ? 0xff - (int)(got & 0xffu) : 0;
                        if (got) atomicAdd(s_count + e, 1);
                        if (out) out[sub] = e;
                    }
                } else {
                    for (int k = 0; k < a.K; ++k) {
                        const uint32_t best = top();
                        if (key[0] == best && best != 0u) {
#pragma unroll
                            for (int j = 0; j < 7; ++j) key[j] = key[j + 1];
                            key[7] = 0u;
                            const int e = 0xff - (int)(best & 0xffu);
                            atomicAdd(s_count + e, 1);
                            if (out) out[k] = e;
                        }
                        if (out && best == 0u && sub == 0) out[k] = 0;
                    }
                }
            } else {
                for (int k = 0; k < a.K; ++k) {
                    uint32_t top = key[0];
#pragma unroll
                    for (int j = 1; j < 8 * NV; ++j) top = max(top, key[j]);
                    uint32_t best = top;
#pragma unroll
                    for (int o = G / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    const uint32_t who = __ballot_sync(0xffffffffu, top == best) & group;
                    if (lane == __ffs(who) - 1) {        // the lowest expert of those that are equal
                        int at = 0;
#pragma unroll
                        for (int j = 8 * NV - 1; j >= 0; --j)
                            if (key[j] == best) at = j;
#pragma unroll
                        for (int j = 0; j < 8 * NV; ++j)
                            if (j == at) key[j] = 0u;
                        const int e = min(e0 + at, a.E - 1);
                        if (valid) atomicAdd(s_count + e, 1);
                        if (out) out[k] = valid ? e : 0;
                    }
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
template <int kType, int NV, int G>
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
    constexpr int kPerWarp = 32 / G, kTurn = kRouterThreads / 32 * kPerWarp;
    const int sub = lane & (G - 1), e0 = sub * 8 * NV;
    const Ty* const base = (const Ty*)a.logits + (long long)it.l * a.stride_l + (a.per_sequence && a.flat_in ? it.b0 * a.stride_b : 0);
    Ty* const dbase = (Ty*)a.dlogits + (long long)it.l * a.dl_stride_l + (a.per_sequence && a.flat_out ? it.b0 * a.dl_stride_b : 0);
    const bool with_z = a.z_coef != 0.f;
    float2 f[4 * NV];                                    // the lane's experts are the same of every token
#pragma unroll
    for (int j = 0; j < 4 * NV; ++j)
        f[j] = make_float2(e0 + 2 * j < a.E ? s_f[e0 + 2 * j] : 0.f, e0 + 2 * j + 1 < a.E ? s_f[e0 + 2 * j + 1] : 0.f);
    // sums of a block's tokens: a lane has some tens of them, added in fp32, then in double
    float sum_dot = 0.f, sum_lse = 0.f;
    int tokens = 0;
    const int mine = warp * kPerWarp + lane / G;
    const int step = a.n_chunks * kTurn;
    int r = it.chunk * kTurn;
    RouterRow w = router_row(a, it, r + mine);
    float z[8 * NV];
    auto load = [&]() {                                  // (a row that is no token has p = 0)
        if (w.valid) {
            router_load<kType, NV>(base + router_at(w, a.flat_in, a.stride_b, a.stride_t), e0, a.E, a.vec_in, -INFINITY, z);
        } else {
#pragma unroll
            for (int j = 0; j < 8 * NV; ++j) z[j] = -INFINITY;
        }
    };
    load();
    for (; r < it.rows; r += step) {
        const bool row = w.row, valid = w.valid;
        Ty* const dst = dbase + router_at(w, a.flat_out, a.dl_stride_b, a.dl_stride_t);
        float2 p[4 * NV], slope[4 * NV];
#pragma unroll
        for (int j = 0; j < 4 * NV; ++j) p[j] = make_float2(z[2 * j], z[2 * j + 1]);
        w = router_row(a, it, r + step + mine);
        load();                                          // in flight meanwhile
        float m = 0.f;
        if (a.scoring == kRouterSoftmax) {
            m = fmaxf(p[0].x, p[0].y);
#pragma unroll
            for (int j = 1; j < 4 * NV; ++j) m = fmaxf(m, fmaxf(p[j].x, p[j].y));
#pragma unroll
            for (int o = G / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (m == -INFINITY) m = 0.f;                 // (no token, or one that may choose no expert)
#pragma unroll
            for (int j = 0; j < 4 * NV; ++j) {
                const float2 y = __fmul2_rn(__fadd2_rn(p[j], splat2(-m)), splat2(kLog2e));
                p[j] = make_float2(ex2(y.x), ex2(y.y));
            }
        } else {
            auto one = [](float v, float& rise) {
                const float e = ex2(-fabsf(v) * kLog2e), inv = __fdividef(1.f, 1.f + e);
                rise = v >= 0.f ? e * inv : inv;
                return v >= 0.f ? inv : e * inv;
            };
#pragma unroll
            for (int j = 0; j < 4 * NV; ++j) {
                p[j].x = one(p[j].x, slope[j].x);
                p[j].y = one(p[j].y, slope[j].y);
            }
        }
        float2 t2 = splat2(0.f), d2 = splat2(0.f);
#pragma unroll
        for (int j = 0; j < 4 * NV; ++j) {
            t2 = __fadd2_rn(t2, p[j]);
            d2 = __ffma2_rn(p[j], f[j], d2);
        }
        float total = t2.x + t2.y, dot = d2.x + d2.y;
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) {
            total += __shfl_xor_sync(0xffffffffu, total, o);
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        const float inv = total > 0.f ? __fdividef(1.f, total) : total;            // (0 stays 0, NaN NaN)
        dot *= inv;
        float lse = 0.f;
        if (with_z && total > 0.f) lse = fmaf(lg2(total), kLn2, m);
        if (row) {
            const float pb = inv * wb, gz = with_z ? inv * wz * lse : 0.f;
            float d[8 * NV];
#pragma unroll
            for (int j = 0; j < 4 * NV; ++j) {
                float2 v = __fadd2_rn(f[j], splat2(-dot));
                if (a.scoring == kRouterSigmoid) v = __fmul2_rn(__fmul2_rn(v, slope[j]), splat2(pb));
                else v = __ffma2_rn(v, splat2(pb), splat2(gz));
                v = __fmul2_rn(v, p[j]);
                d[2 * j] = v.x;
                d[2 * j + 1] = v.y;
            }
            router_store<kType, NV>(dst, e0, a.E, a.vec_out, d);
        }
        if (valid && sub == 0) {
            if (total != 0.f) {                          // (0: a token that may choose no expert)
                sum_dot += dot;
                ++tokens;
            }
            sum_lse = fmaf(lse, lse, sum_lse);
        }
    }
    double sum_b = (double)tokens + (double)sum_dot, sum_z = (double)sum_lse;
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
