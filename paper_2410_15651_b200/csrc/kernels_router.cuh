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
// Two launches: counts, then losses and gradient.  A token is held by G = 1 .. 32 lanes with one vector of eight entries each, or
// two (16-bit logits of more than 8 experts) or four (above 512 experts); the rows are dealt to the blocks in turns, so that the
// padding of short sequences is shared out.  Large calls read the logits twice and write the gradient once; what bounds them is
// the selection and the softmax themselves (24 layers x 16 x 1024 tokens x 128 experts, K = 8, bf16, half of them padding: 119 us
// for 189 MB, 1.6 TB/s; both kernels issue in about 45 % of the cycles, three blocks a multiprocessor).  Small calls are bound by
// their two launches (23 us with the host's share at 2 x 16 tokens of 8 experts, 22 us at 16 x 1024 of 256 in fp32).
// Two vectors per lane halve the shuffles of a token (176 -> 148 us), and as many blocks as are resident at once spare the
// later ones' start and the last ones' wait (1184 blocks 143 us, 888 123 us, 592 147 us, 444 119 us).
#pragma once
#include "common.cuh"

namespace rlhf {

constexpr int kRouterThreads = 256;
constexpr int kRouterMaxExperts = 1024;
constexpr int kRouterMaxChunks = 256;        // chunks of a group (partial counts: one per kRouterCluster of them)
constexpr int kRouterCluster = 8;
constexpr int kRouterTargetBlocks = 444;     // three a multiprocessor, all of them at once

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
template <> struct RouterEl<0> { using T = uint16_t; };
template <> struct RouterEl<1> { using T = uint16_t; };
template <> struct RouterEl<2> { using T = float; };

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

// A lane has NV vectors of eight entries, sub, sub + G and so on of its token's (neighbours in one access).  Its entries come in
// pairs; the first expert of pair j:
template <int G>
__device__ __forceinline__ int router_expert(int sub, int j) { return 8 * (sub + G * (j >> 2)) + 2 * (j & 3); }

// A lane's entries as they lie; `missing` past E.
template <int kType, int NV, int G>
struct RouterRaw {
    using Ty = typename RouterEl<kType>::T;
    static constexpr bool kHalf = sizeof(Ty) == 2;
    uint32_t w[(kHalf ? 4 : 8) * NV];

    __device__ __forceinline__ void fill(uint32_t missing)
    {
#pragma unroll
        for (int j = 0; j < (kHalf ? 4 : 8) * NV; ++j) w[j] = missing;
    }
    __device__ __forceinline__ void load(const Ty* row, int sub, int E, bool vec, uint32_t missing)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int e = router_expert<G>(sub, 4 * v);
            uint32_t* o = w + (kHalf ? 4 : 8) * v;
            if (vec) {                       // E is a multiple of 8 then
                uint4 q = make_uint4(missing, missing, missing, missing), x = q;
                if (e < E) {
                    q = __ldg((const uint4*)(row + e));
                    if (!kHalf) x = __ldg((const uint4*)(row + e) + 1);
                }
                o[0] = q.x; o[1] = q.y; o[2] = q.z; o[3] = q.w;
                if (!kHalf) { o[4] = x.x; o[5] = x.y; o[6] = x.z; o[7] = x.w; }
            } else if constexpr (kHalf) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o[j] = (e + 2 * j < E ? (uint32_t)row[e + 2 * j] : missing & 0xffffu) |
                           (e + 2 * j + 1 < E ? (uint32_t)row[e + 2 * j + 1] << 16 : missing & 0xffff0000u);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = e + j < E ? __float_as_uint(row[e + j]) : missing;
            }
        }
    }
    __device__ __forceinline__ float2 pair(int j) const
    {
        if constexpr (kHalf) return El<kType == 1>::unpack2(w[j]);
        else return make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
    }
    static __device__ __forceinline__ uint32_t minus_inf() { return kType == 0 ? 0xff80ff80u : kType == 1 ? 0xfc00fc00u : 0xff800000u; }
};

template <int kType, int NV, int G>
__device__ __forceinline__ void router_store(typename RouterEl<kType>::T* row, int sub, int E, bool vec, const float2 (&d)[4 * NV])
{
    using Ty = typename RouterEl<kType>::T;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = router_expert<G>(sub, 4 * v);
        const float2* x = d + 4 * v;
        if constexpr (sizeof(Ty) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = El<kType == 1>::pack2(x[j].x, x[j].y);
            if (vec) {
                if (e < E) __stcs((uint4*)(row + e), make_uint4(w[0], w[1], w[2], w[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e + j < E) row[e + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            }
        } else {
            if (vec) {
                if (e < E) {
                    __stcs((float4*)(row + e), make_float4(x[0].x, x[0].y, x[1].x, x[1].y));
                    __stcs((float4*)(row + e) + 1, make_float4(x[2].x, x[2].y, x[3].x, x[3].y));
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e + j < E) row[e + j] = j & 1 ? x[j >> 1].y : x[j >> 1].x;
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

// Lanes of a token with nv vectors each.
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
        // 16-bit logits of up to 256 experts: a key orders logit and expert at once (the higher logit, then the lower expert).  A lane
        // sorts its own, and each choice is the largest head of the token's lanes.  Else a choice looks through all.
        constexpr int N = 8 * NV;
        constexpr bool kSorted = sizeof(Ty) == 2 && N * G <= 256;
        constexpr int kPerWarp = 32 / G, kTurn = kRouterThreads / 32 * kPerWarp;
        const int sub = lane & (G - 1);
        const Ty* const base = (const Ty*)a.logits + (long long)it.l * a.stride_l + (a.per_sequence && a.flat_in ? it.b0 * a.stride_b : 0);
        int* const ids_base = a.out_ids + ((long long)it.l * a.B + it.b0) * a.T * a.K;
        const int mine = warp * kPerWarp + lane / G;
        const int step = a.n_chunks * kTurn;
        int r = it.chunk * kTurn;
        RouterRow w = router_row(a, it, r + mine);
        RouterRaw<kType, NV, G> z;
        z.fill(0u);
        auto load = [&]() {
            if (w.valid) z.load(base + router_at(w, a.flat_in, a.stride_b, a.stride_t), sub, a.E, a.vec_in, 0u);
        };
        load();
        // (every lane of a warp makes every turn: the shuffles want them all)
        for (; r < it.rows; r += step) {
            const bool valid = w.valid;
            int* const out = a.out_ids && w.row ? ids_base + (long long)w.r * a.K : nullptr;
            uint32_t key[N];
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const int e = router_expert<G>(sub, j);
                if constexpr (kSorted) {
                    const uint32_t x = router_order2<kType == 1>(z.w[j]);
                    key[2 * j] = (x << 16) + (0xffffu - (uint32_t)e);
                    key[2 * j + 1] = (x & 0xffff0000u) | (0xfffeu - (uint32_t)e);
                } else {
                    const float2 x = z.pair(j);
                    key[2 * j] = router_key(x.x);
                    key[2 * j + 1] = router_key(x.y);
                }
                if (!valid || e >= a.E) key[2 * j] = 0u;
                if (!valid || e + 1 >= a.E) key[2 * j + 1] = 0u;
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
#pragma unroll
                for (int i = 0; i < N; i += 8) {         // Batcher's odd-even merge of eight
                    order(i, i + 1); order(i + 2, i + 3); order(i + 4, i + 5); order(i + 6, i + 7);
                    order(i, i + 2); order(i + 1, i + 3); order(i + 4, i + 6); order(i + 5, i + 7);
                    order(i + 1, i + 2); order(i + 5, i + 6);
                    order(i, i + 4); order(i + 1, i + 5); order(i + 2, i + 6); order(i + 3, i + 7);
                    order(i + 2, i + 4); order(i + 3, i + 5);
                    order(i + 1, i + 2); order(i + 3, i + 4); order(i + 5, i + 6);
                }
                auto bitonic = [&](int i) {              // sorts eight that rise and fall
                    order(i, i + 4); order(i + 1, i + 5); order(i + 2, i + 6); order(i + 3, i + 7);
                    order(i, i + 2); order(i + 1, i + 3); order(i + 4, i + 6); order(i + 5, i + 7);
                    order(i, i + 1); order(i + 2, i + 3); order(i + 4, i + 5); order(i + 6, i + 7);
                };
                auto top = [&]() {
                    uint32_t best = key[0];
#pragma unroll
                    for (int o = G / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    return best;
                };
                if (a.K <= 8) {                          // lane k % G of a token keeps its k-th choice
                    if constexpr (NV == 2) {             // (eight of sixteen will do)
#pragma unroll
                        for (int i = 0; i < 8; ++i) key[i] = max(key[i], key[15 - i]);
                        bitonic(0);
                    }
                    uint32_t got[8 / (G < 8 ? G : 8)];
#pragma unroll
                    for (int i = 0; i < 8 / (G < 8 ? G : 8); ++i) got[i] = 0u;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (k >= a.K) break;
                        const uint32_t best = top();
                        const bool won = key[0] == best;
                        if (sub == (k & (G - 1))) got[k / G] = best;
#pragma unroll
                        for (int j = 0; j < 7 - k; ++j) key[j] = won ? key[j + 1] : key[j];
                    }
#pragma unroll
                    for (int i = 0; i < 8 / (G < 8 ? G : 8); ++i) {
                        const int k = i * G + sub;
                        if (k < a.K) {
                            const int e = got[i] ? 0xff - (int)(got[i] & 0xffu) : 0;
                            if (got[i]) atomicAdd(s_count + e, 1);
                            if (out) out[k] = e;
                        }
                    }
                } else {
                    if constexpr (NV == 2) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {    // the upper eight, the lower eight
                            const uint32_t x = key[i], y = key[15 - i];
                            key[i] = max(x, y);
                            key[15 - i] = min(x, y);
                        }
                        bitonic(0);
                        bitonic(8);
                    }
                    for (int k = 0; k < a.K; ++k) {
                        const uint32_t best = top();
                        if (key[0] == best && best != 0u) {
#pragma unroll
                            for (int j = 0; j < N - 1; ++j) key[j] = key[j + 1];
                            key[N - 1] = 0u;
                            const int e = 0xff - (int)(best & 0xffu);
                            atomicAdd(s_count + e, 1);
                            if (out) out[k] = e;
                        }
                        if (out && best == 0u && sub == 0) out[k] = 0;
                    }
                }
            } else {
                for (int k = 0; k < a.K; ++k) {
                    uint32_t best = key[0];
#pragma unroll
                    for (int j = 1; j < N; ++j) best = max(best, key[j]);
#pragma unroll
                    for (int o = G / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    int e = kRouterMaxExperts;           // the lowest expert of those that are equal
#pragma unroll
                    for (int j = N - 1; j >= 0; --j)
                        if (key[j] == best) e = router_expert<G>(sub, j >> 1) + (j & 1);
#pragma unroll
                    for (int o = G / 2; o > 0; o >>= 1) e = min(e, __shfl_xor_sync(0xffffffffu, e, o));
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (e == router_expert<G>(sub, j >> 1) + (j & 1)) key[j] = 0u;
                    if (sub == 0) {
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
__global__ void __launch_bounds__(kRouterThreads, NV == 1 ? 4 : NV == 2 ? 3 : 1) router_loss_kernel(const __grid_constant__ RouterArgs a)
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
    const int sub = lane & (G - 1);
    const Ty* const base = (const Ty*)a.logits + (long long)it.l * a.stride_l + (a.per_sequence && a.flat_in ? it.b0 * a.stride_b : 0);
    Ty* const dbase = (Ty*)a.dlogits + (long long)it.l * a.dl_stride_l + (a.per_sequence && a.flat_out ? it.b0 * a.dl_stride_b : 0);
    const bool with_z = a.z_coef != 0.f;
    float2 f[4 * NV];                                    // the lane's experts are the same of every token
#pragma unroll
    for (int j = 0; j < 4 * NV; ++j) {
        const int e = router_expert<G>(sub, j);
        f[j] = make_float2(e < a.E ? s_f[e] : 0.f, e + 1 < a.E ? s_f[e + 1] : 0.f);
    }
    // sums of a block's tokens: a lane has some tens of them, added in fp32, then in double
    float sum_dot = 0.f, sum_lse = 0.f;
    int tokens = 0;
    const int mine = warp * kPerWarp + lane / G;
    const int step = a.n_chunks * kTurn;
    int r = it.chunk * kTurn;
    RouterRow w = router_row(a, it, r + mine);
    RouterRaw<kType, NV, G> z;
    auto load = [&]() {                                  // (a row that is no token has p = 0)
        if (w.valid) z.load(base + router_at(w, a.flat_in, a.stride_b, a.stride_t), sub, a.E, a.vec_in, z.minus_inf());
        else z.fill(z.minus_inf());
    };
    load();
    for (; r < it.rows; r += step) {
        const bool row = w.row, valid = w.valid;
        Ty* const dst = dbase + router_at(w, a.flat_out, a.dl_stride_b, a.dl_stride_t);
        float2 p[4 * NV], slope[4 * NV];
#pragma unroll
        for (int j = 0; j < 4 * NV; ++j) p[j] = z.pair(j);
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
#pragma unroll
            for (int j = 0; j < 4 * NV; ++j) {
                float2 v = __fadd2_rn(f[j], splat2(-dot));
                if (a.scoring == kRouterSigmoid) v = __fmul2_rn(__fmul2_rn(v, slope[j]), splat2(pb));
                else v = __ffma2_rn(v, splat2(pb), splat2(gz));
                p[j] = __fmul2_rn(v, p[j]);
            }
            router_store<kType, NV, G>(dst, sub, a.E, a.vec_out, p);
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
