// The K largest log-probs of every row of a logits tensor, for rows of any alignment.
//
// One block per row, rows dealt from a counter in the workspace.  The row is streamed once: every thread keeps an online
// partition sum (running maximum and sum, fp32) and the maxima of eight groups of its vectors (vector j of a thread
// belongs to group j mod 8).  The K-th largest of the 8 * threads group maxima is a lower bound of the K-th largest entry
// -- K groups hold an entry at least that large -- and, the groups being many, a tight one: with G groups about
// -G ln(1 - K/G) entries reach it (65 for K = 64, 2048 groups), so that only the groups above it, some K of them, are read
// again (from L2) to collect the candidates, and the candidates are ranked by counting the larger ones.  Candidates are
// compared as (value, lower index first), so the result does not depend on the order in which they were collected.
// Rows with more candidates than the list holds (long runs of equal values, rows sorted against the groups) are selected
// by bisection over the 16-bit values with repeated reads of the row, ties in index order.
//
// Exponents are formed as (z - maximum) * log2(e) / temperature: the difference of two 16-bit values is exact or nearly so,
// whatever their size.
//
// Bound: one read of the row from DRAM; per logit one ex2 and half a packed maximum.
#pragma once
#include "kernels_ring.cuh"

namespace rlhf {

constexpr int kTopkMax = 256;
constexpr int kTopkGroups = 8;          // per thread
constexpr int kTopkCandidates = 2048;
constexpr float kTopkFloor = -3.0e38f;  // maximum of a thread that has seen no entry

struct TopkArgs {
    const uint16_t* logits;
    long long stride_b, stride_t;
    const int* lengths;
    int B, T, V, K;
    float scale;                // log2(e) / temperature
    int* ids;                   // [B,T,K]
    float* logprobs;            // [B,T,K]
    unsigned* status;
    unsigned* ticket;           // workspace words, zero between calls
    unsigned* row_counter;
};

// Order of the 16-bit values as whole numbers: -0 and +0 equal, NaN above everything with its sign.
__device__ __forceinline__ uint32_t order_key(uint32_t bits16)
{
    return (bits16 & 0x8000u) ? 0x8000u - (bits16 & 0x7fffu) : 0x8000u + bits16;
}
__device__ __forceinline__ uint32_t key_bits(uint32_t key) { return key >= 0x8000u ? key - 0x8000u : 0x8000u | (0x8000u - key); }
template <bool kF16>
__device__ __forceinline__ uint32_t key_of_neg_inf() { return order_key(El<kF16>::kNegInf); }

template <bool kF16>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    uint32_t r;
    if (kF16) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// A row as the 16-byte aligned span that holds it.
struct RowSpan {
    const uint4* vecs;
    uint32_t eoff;              // entries of the first vector that precede the row
    uint32_t nvec;
    uint32_t tail;              // entries of the last vector that belong to the row (1..8, counted from the vector's start)
};

__device__ __forceinline__ RowSpan row_span(const uint16_t* row, int V)
{
    RowSpan r;
    const uint32_t mis = (uint32_t)((uintptr_t)row & 15u);
    r.vecs = (const uint4*)((const unsigned char*)row - mis);
    r.eoff = mis >> 1;
    r.nvec = (r.eoff + (uint32_t)V + 7u) >> 3;
    r.tail = r.eoff + (uint32_t)V - 8u * (r.nvec - 1u);
    return r;
}

__device__ __forceinline__ uint4 load_streaming(const uint4* p)
{
    uint4 q;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}

// Vector v of the span, entries that are not the row's replaced by -inf.
template <bool kF16>
__device__ __forceinline__ uint4 span_vec(const RowSpan& r, uint32_t v)
{
    uint4 q = load_streaming(r.vecs + v);
    if (v == 0 || v == r.nvec - 1)
        q = mask_vec_outside<kF16>(q, v == 0 ? (int)r.eoff : 0, v == r.nvec - 1 ? (int)r.tail : 8);
    return q;
}

// Sum of one unsigned per thread, for every thread; `scratch` holds two sets of NT/32 words, used alternately.
template <int NT>
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t* scratch, int& turn)
{
    uint32_t* s = scratch + (turn ^= 1) * (NT / 32);
    v = __reduce_add_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) t += s[w];
    return t;
}

__device__ __forceinline__ unsigned long long candidate(uint32_t key, uint32_t index)
{
    return ((unsigned long long)key << 32) | (0xffffffffu - index);
}

// Appends the entries of vector v with a key of at least `least`.
template <bool kF16>
__device__ __forceinline__ void collect_vec(const RowSpan& r, uint32_t v, uint32_t least, unsigned long long* cand, uint32_t* n_cand)
{
    const uint4 q = span_vec<kF16>(r, v);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t key = order_key((i & 1) ? (w[i >> 1] >> 16) : (w[i >> 1] & 0xffffu));
        if (key >= least) {
            const uint32_t at = atomicAdd(n_cand, 1u);
            if (at < (uint32_t)kTopkCandidates) cand[at] = candidate(key, v * 8u + (uint32_t)i - r.eoff);
        }
    }
}

template <int NT, bool kF16>
__device__ __forceinline__ uint32_t count_at_least(const RowSpan& r, uint32_t least, uint32_t* scratch, int& turn)
{
    uint32_t n = 0;
    for (uint32_t v = threadIdx.x; v < r.nvec; v += NT) {
        const uint4 q = span_vec<kF16>(r, v);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) n += order_key((i & 1) ? (w[i >> 1] >> 16) : (w[i >> 1] & 0xffffu)) >= least ? 1u : 0u;
    }
    return block_sum<NT>(n, scratch, turn);
}

// Selection without the candidate bound: the largest key that K entries reach, found by bisection, then the entries above
// it and, in index order, as many of the entries equal to it as are missing.  Whole block; returns the candidates.
template <int NT, bool kF16>
__device__ __noinline__ uint32_t topk_bisect(const RowSpan& r, uint32_t K, unsigned long long* cand, uint32_t* n_cand,
                                             uint32_t* scratch, int& turn)
{
    uint32_t lo = key_of_neg_inf<kF16>() + 1u, hi = 65536u;
    const bool few = count_at_least<NT, kF16>(r, lo, scratch, turn) <= K;
    while (!few && hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (count_at_least<NT, kF16>(r, mid, scratch, turn) >= K) lo = mid; else hi = mid;
    }
    if (threadIdx.x == 0) *n_cand = 0;
    __syncthreads();
    for (uint32_t v = threadIdx.x; v < r.nvec; v += NT) collect_vec<kF16>(r, v, few ? lo : lo + 1u, cand, n_cand);
    __syncthreads();
    uint32_t n = min(*n_cand, (uint32_t)kTopkCandidates);
    if (few) return n;
    // entries equal to `lo`, in index order
    for (uint32_t v0 = 0; v0 < r.nvec && n < K; v0 += NT) {
        const uint32_t v = v0 + threadIdx.x;
        uint32_t hit = 0;
        if (v < r.nvec) {
            const uint4 q = span_vec<kF16>(r, v);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (order_key((i & 1) ? (w[i >> 1] >> 16) : (w[i >> 1] & 0xffffu)) == lo) hit |= 1u << i;
        }
        const uint32_t mine = (uint32_t)__popc(hit);
        uint32_t upto = mine;                                    // inclusive prefix within the warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if ((int)(threadIdx.x & 31) >= o) upto += x;
        }
        uint32_t* s = scratch + (turn ^= 1) * (NT / 32);
        if ((threadIdx.x & 31) == 31) s[threadIdx.x >> 5] = upto;
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int w = 0; w < NT / 32; ++w) {
            if (w < (int)(threadIdx.x >> 5)) before += s[w];
            all += s[w];
        }
        uint32_t at = n + before + upto - mine;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((hit >> i) & 1u) {
                if (at < K) cand[at] = candidate(lo, v * 8u + (uint32_t)i - r.eoff);
                ++at;
            }
        n = min(K, n + all);
    }
    __syncthreads();
    return n;
}

// NT threads per row; as many blocks per SM as registers allow, so that some stream while others select.
template <int NT, bool kF16>
__global__ void __launch_bounds__(NT, NT >= 1024 ? 1 : 1024 / NT) topk_logprobs_kernel(TopkArgs p)
{
    constexpr int kWarps = NT / 32;
    __shared__ unsigned long long s_cand[kTopkCandidates];
    __shared__ uint16_t s_group[kTopkGroups * NT];
    __shared__ uint32_t s_scratch[2 * kWarps];
    __shared__ float2 s_part[kWarps];
    __shared__ uint32_t s_lo[kWarps], s_hi[kWarps];
    __shared__ uint32_t s_n[2];                     // qualifying groups, candidates
    __shared__ long long s_row[2];
    __shared__ long long s_cnt[33];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int turn = 0;

    pdl_wait_prior_grid();
    pdl_release_next_grid();
    if (blockIdx.x == 0) block_count_valid(p.lengths, p.B, p.T, s_cnt, p.status);
    const long long total = (long long)p.B * p.T;
    const uint32_t empty = key_of_neg_inf<kF16>();
    if (tid == 0) s_row[0] = (long long)atomicAdd(p.row_counter, 1u);

    for (int i = 0;; ++i) {
        __syncthreads();                            // s_row[i & 1] is there; the previous row's shared data has been read
        const long long row = s_row[i & 1];
        if (row >= total) break;
        if (tid == 0) {
            s_row[(i + 1) & 1] = (long long)atomicAdd(p.row_counter, 1u);   // the next row, in flight during this one
            s_n[0] = s_n[1] = 0;
        }
        const int b = (int)(row / p.T), t = (int)(row % p.T);
        int* ids = p.ids + row * p.K;
        float* lps = p.logprobs + row * p.K;
        if (t >= clamp_len(__ldg(p.lengths + b), p.T)) {
            for (int k = tid; k < p.K; k += NT) { ids[k] = 0; lps[k] = 0.f; }
            continue;
        }
        const RowSpan r = row_span(p.logits + (long long)b * p.stride_b + (long long)t * p.stride_t, p.V);

        // ---- the stream: partition sum and group maxima
        uint32_t g2[kTopkGroups];
#pragma unroll
        for (int u = 0; u < kTopkGroups; ++u) g2[u] = El<kF16>::kNegInf2;
        float zm = kTopkFloor, s = 0.f;             // running maximum and sum of 2^((z - zm) * scale)
        for (uint32_t v0 = tid; v0 < r.nvec; v0 += kTopkGroups * NT) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 q[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t v = v0 + (4 * h + u) * NT;
                    q[u] = make_uint4(El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2);
                    if (v < r.nvec) q[u] = load_streaming(r.vecs + v);
                }
                uint32_t m2 = El<kF16>::kNegInf2;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t v = v0 + (4 * h + u) * NT;
                    if (v == 0 || v == r.nvec - 1)
                        q[u] = mask_vec_outside<kF16>(q[u], v == 0 ? (int)r.eoff : 0, v == r.nvec - 1 ? (int)r.tail : 8);
                    const uint32_t vm = max2<kF16>(max2<kF16>(q[u].x, q[u].y), max2<kF16>(q[u].z, q[u].w));
                    g2[4 * h + u] = max2<kF16>(g2[4 * h + u], vm);
                    m2 = max2<kF16>(m2, vm);
                }
                const float2 mf = El<kF16>::unpack2(m2);
                const float zn = fmaxf(zm, fmaxf(mf.x, mf.y));
                float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 x = __fmul2_rn(__fadd2_rn(El<kF16>::unpack2(w[k]), splat2(-zn)), splat2(p.scale));
                        acc[k & 1] = __fadd2_rn(acc[k & 1], make_float2(ex2(x.x), ex2(x.y)));
                    }
                }
                s = fmaf(s, ex2((zm - zn) * p.scale), (acc[0].x + acc[0].y) + (acc[1].x + acc[1].y));
                zm = zn;
            }
        }

        // ---- block totals: the row's maximum and sum; smallest and largest group maximum
        uint32_t key[kTopkGroups], lo = 65535u, hi = 0u;
#pragma unroll
        for (int u = 0; u < kTopkGroups; ++u) {
            key[u] = max(order_key(g2[u] & 0xffffu), order_key(g2[u] >> 16));
            if (key[u] <= empty) key[u] = 0;                       // nothing in it to select
            hi = max(hi, key[u]);
            lo = min(lo, key[u]);
        }
        float zw = zm;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) zw = fmaxf(zw, __shfl_xor_sync(0xffffffffu, zw, o));
        float sw = s * ex2((zm - zw) * p.scale);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sw += __shfl_xor_sync(0xffffffffu, sw, o);
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) { s_part[warp] = make_float2(zw, sw); s_lo[warp] = lo; s_hi[warp] = hi; }
        __syncthreads();
        float zt = kTopkFloor, st = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { zt = fmaxf(zt, s_part[w].x); lo = min(lo, s_lo[w]); hi = max(hi, s_hi[w]); }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) st += s_part[w].y * ex2((s_part[w].x - zt) * p.scale);
        const float l2 = log2f(st);

        // ---- the K-th largest group maximum, by trisection (two counts of at most 2^14 in one reduction)
        lo = max(lo, empty + 1u);                                  // every selectable entry reaches this
        uint32_t end = hi + 1u;                                    // nothing reaches this
        bool enough = true;
        {
            uint32_t n = 0;
#pragma unroll
            for (int u = 0; u < kTopkGroups; ++u) n += key[u] >= lo ? 1u : 0u;
            enough = block_sum<NT>(n, s_scratch, turn) >= (uint32_t)p.K;
        }
        while (enough && end - lo > 1u) {
            const uint32_t d = end - lo, p1 = lo + max(1u, d / 3u), p2 = max(p1, lo + 2u * d / 3u);
            uint32_t n = 0;
#pragma unroll
            for (int u = 0; u < kTopkGroups; ++u) n += (key[u] >= p1 ? 1u : 0u) + (key[u] >= p2 ? 65536u : 0u);
            n = block_sum<NT>(n, s_scratch, turn);
            if ((n >> 16) >= (uint32_t)p.K) lo = p2;
            else if ((n & 0xffffu) >= (uint32_t)p.K) { lo = p1; end = p2; }      // p1 < p2 here: their counts differ
            else end = p1;
        }

        // ---- the groups that reach it, and their entries that do
#pragma unroll
        for (int u = 0; u < kTopkGroups; ++u)
            if (key[u] >= lo) s_group[atomicAdd(&s_n[0], 1u)] = (uint16_t)(u * NT + tid);
        __syncthreads();
        const uint32_t rounds = (r.nvec + kTopkGroups * NT - 1) / (kTopkGroups * NT), items = s_n[0] * rounds;
        for (uint32_t it = tid; it < items; it += NT) {
            const uint32_t v = s_group[it / rounds] + (it % rounds) * (kTopkGroups * NT);
            if (v < r.nvec) collect_vec<kF16>(r, v, lo, s_cand, &s_n[1]);
        }
        __syncthreads();
        uint32_t n = s_n[1];
        if (n > (uint32_t)kTopkCandidates) n = topk_bisect<NT, kF16>(r, (uint32_t)p.K, s_cand, &s_n[1], s_scratch, turn);

        // ---- ranks: the number of larger candidates
        for (uint32_t c = tid; c < n; c += NT) {
            const unsigned long long mine = s_cand[c];
            uint32_t rank = 0;
            for (uint32_t o = 0; o < n; ++o) rank += s_cand[o] > mine ? 1u : 0u;
            if (rank < (uint32_t)p.K) {
                const float z = El<kF16>::widen(key_bits((uint32_t)(mine >> 32)));
                ids[rank] = (int)(0xffffffffu - (uint32_t)mine);
                lps[rank] = kLn2 * fmaf(z - zt, p.scale, -l2);
            }
        }
        for (uint32_t k = n + tid; k < (uint32_t)p.K; k += NT) {    // fewer entries than K
            ids[k] = -1;
            lps[k] = __uint_as_float(0xff800000u);
        }
    }
    if (tid == 0) {
        if (atomicAdd(p.ticket, 1u) == gridDim.x - 1) { *p.ticket = 0u; *p.row_counter = 0u; }
    }
}

}  // namespace rlhf
