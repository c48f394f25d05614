// The K largest log-probs of every row of a logits tensor, for rows of any alignment.
//
// A row is streamed once: every thread keeps an online partition sum (running maximum and sum, fp32) and the maxima of
// groups of the entries that it sees.  The K-th largest of G group maxima is a lower bound of the K-th largest entry -- K
// groups hold an entry at least that large -- and a tight one: of random entries about -G ln(1 - K/G) reach it (74 for
// K = 64, G = 256).  Only the groups that reach it are read again, to collect the candidates.  Candidates are compared as
// (value, lower index first), so the result does not depend on the order in which they were collected.
//
// One block per row, several blocks per SM, rows dealt from a counter in the workspace.
//
// Exponents are formed as (z - maximum) * log2(e) / temperature: the difference of two 16-bit values is exact or nearly so,
// whatever their size.
//
// Floor: one read of the row from DRAM (32 us for 2048 rows of 50272 in bf16 at 6.5 TB/s).  Nothing is full: DRAM 45%, issue slots
// 48%, and a warp waits 6.9 of 14.1 cycles per instruction for global loads.  Too few rows are streamed at a time: a block that
// selects a row loads nothing new, and at 64 registers an SM holds 1024 threads.  The same rows of 50272 take 1.8 times as long
// at K = 256 as at K = 64 (candidates are ranked pair by pair), and 0.8 times at K = 8.  Fewer registers for more blocks per SM, and
// a sort of the candidates, are not tried.  Per row and K = 64 there are 14,600 warp
// instructions, some 9,000 of them for the stream (one ex2 and half a packed maximum per logit).  Measured on such rows and
// dropped, with their time over this kernel's: the first 8 to 32 KB of the next row brought to L2 before the selection (0.99
// to 1.03, and 1.04 at V = 1000); a row per warp (all rows of a batch are then in flight, L2 does not hold
// them, and what is read again comes from DRAM in sectors: 1.43; with groups of whole lines 0.93, but 1.13 at K = 256 and
// 1.18 at V = 128256); separate streaming and selecting warps (1.25: one warp selects for 25 us); rows through a ring of
// bulk copies (1.05).
#pragma once
#include "kernels_ring.cuh"
#include <cuda_fp16.h>

namespace rlhf {

constexpr int kTopkMax = 256;
constexpr int kTopkGroups = 8;          // per thread
constexpr int kTopkCandidates = 1024;
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

// ---------------------------------------------------------------- order and candidates
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

// ---------------------------------------------------------------- rows
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

// Entry i of a vector.
__device__ __forceinline__ uint32_t vec_entry(const uint4& q, int i)
{
    const uint32_t w = (i >> 1) == 0 ? q.x : ((i >> 1) == 1 ? q.y : ((i >> 1) == 2 ? q.z : q.w));
    return (i & 1) ? (w >> 16) : (w & 0xffffu);
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

// Barrier over the NT threads that work on a row; the second form also counts those with a predicate.
template <int NT>
__device__ __forceinline__ void row_sync() { asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory"); }
template <int NT>
__device__ __forceinline__ int row_count(bool x)
{
    int n;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.popc.u32 %0, 1, %2, q;\n\t}" : "=r"(n) : "r"((uint32_t)x), "n"(NT) : "memory");
    return n;
}

// Sum of one unsigned per thread, for every thread; `scratch` holds two sets of NT/32 words, used alternately.
template <int NT>
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t* scratch, int& turn)
{
    uint32_t* s = scratch + (turn ^= 1) * (NT / 32);
    v = __reduce_add_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    row_sync<NT>();
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) t += s[w];
    return t;
}

__device__ __forceinline__ unsigned long long candidate(uint32_t key, uint32_t index)
{
    return ((unsigned long long)key << 32) | (0xffffffffu - index);
}

// Two lanes of 16 bits: all ones where a >= b (or a == b), as numbers (never for NaN).
template <bool kF16, bool kEqual>
__device__ __forceinline__ uint32_t mask2(uint32_t a, uint32_t b)
{
    if (kF16) return kEqual ? __heq2_mask(*(const __half2*)&a, *(const __half2*)&b) : __hge2_mask(*(const __half2*)&a, *(const __half2*)&b);
    return kEqual ? __heq2_mask(*(const __nv_bfloat162*)&a, *(const __nv_bfloat162*)&b)
                  : __hge2_mask(*(const __nv_bfloat162*)&a, *(const __nv_bfloat162*)&b);
}

// Bit e: entry e of the vector has a key of at least (kEqual: equal to) that of the value in both halves of `least2`.
template <bool kF16, bool kEqual>
__device__ __forceinline__ uint32_t entries_that_reach(const uint4& q, uint32_t least2)
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t hit = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t m = mask2<kF16, kEqual>(w[k], least2);
        hit |= (m & (1u << (2 * k))) | ((m >> 16) & (2u << (2 * k)));
    }
    return hit;
}
__device__ __forceinline__ uint32_t both_halves(uint32_t key) { return key_bits(key) * 0x10001u; }

// Appends the entries of vector v, whose bits are q, with a key of at least `least`.
template <bool kF16>
__device__ __forceinline__ void collect_entries(const RowSpan& r, const uint4& q, uint32_t v, uint32_t least, unsigned long long* cand, uint32_t* n_cand)
{
    uint32_t hit = entries_that_reach<kF16, false>(q, both_halves(least));
    if (!hit) return;
    uint32_t at = atomicAdd(n_cand, (uint32_t)__popc(hit));
    while (hit) {
        const int i = __ffs(hit) - 1;
        hit &= hit - 1;
        if (at < (uint32_t)kTopkCandidates) cand[at] = candidate(order_key(vec_entry(q, i)), v * 8u + (uint32_t)i - r.eoff);
        ++at;
    }
}

template <bool kF16>
__device__ __forceinline__ void collect_vec(const RowSpan& r, uint32_t v, uint32_t least, unsigned long long* cand, uint32_t* n_cand)
{
    collect_entries<kF16>(r, span_vec<kF16>(r, v), v, least, cand, n_cand);
}

template <int NT, bool kF16>
__device__ __forceinline__ uint32_t count_at_least(const RowSpan& r, uint32_t least, uint32_t* scratch, int& turn)
{
    uint32_t n = 0;
    for (uint32_t v = threadIdx.x; v < r.nvec; v += NT) {
        n += (uint32_t)__popc(entries_that_reach<kF16, false>(span_vec<kF16>(r, v), both_halves(least)));
    }
    return block_sum<NT>(n, scratch, turn);
}

// Selection without the candidate bound: the largest key that K entries reach, found by bisection, then the entries above
// it and, in index order, as many of the entries equal to it as are missing.  Whole block; returns the candidates.
template <int NT, bool kF16>
__device__ __noinline__ uint32_t topk_bisect(const RowSpan& r, uint32_t K, unsigned long long* cand, uint32_t* n_cand,
                                             uint32_t* scratch, int& turn)
{
    uint32_t lo = key_of_neg_inf<kF16>() + 1u, hi = 65536u - key_of_neg_inf<kF16>() + 1u;   // above +inf
    const bool few = count_at_least<NT, kF16>(r, lo, scratch, turn) <= K;
    while (!few && hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (count_at_least<NT, kF16>(r, mid, scratch, turn) >= K) lo = mid; else hi = mid;
    }
    if (threadIdx.x == 0) *n_cand = 0;
    row_sync<NT>();
    for (uint32_t v = threadIdx.x; v < r.nvec; v += NT) collect_vec<kF16>(r, v, few ? lo : lo + 1u, cand, n_cand);
    row_sync<NT>();
    uint32_t n = min(*n_cand, (uint32_t)kTopkCandidates);
    if (few) return n;
    // entries equal to `lo`, in index order
    for (uint32_t v0 = 0; v0 < r.nvec && n < K; v0 += NT) {
        const uint32_t v = v0 + threadIdx.x;
        uint32_t hit = 0;
        if (v < r.nvec) hit = entries_that_reach<kF16, true>(span_vec<kF16>(r, v), both_halves(lo));
        const uint32_t mine = (uint32_t)__popc(hit);
        uint32_t upto = mine;                                    // inclusive prefix within the warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if ((int)(threadIdx.x & 31) >= o) upto += x;
        }
        uint32_t* s = scratch + (turn ^= 1) * (NT / 32);
        if ((threadIdx.x & 31) == 31) s[threadIdx.x >> 5] = upto;
        row_sync<NT>();
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
    row_sync<NT>();
    return n;
}

// One thread's part of a row that NT threads stream: group maxima (two values each), running maximum and sum of
// 2^((z - zm) * scale).  The vectors that lie inside the row belong to groups; the first and the last, which may hold
// entries of neighbouring rows, are added to the sums of one thread each and belong to none.
template <int NT, bool kF16>
__device__ __forceinline__ void stream_row(const RowSpan& r, int tid, float scale, uint32_t (&g2)[kTopkGroups], float& zm, float& s)
{
#pragma unroll
    for (int u = 0; u < kTopkGroups; ++u) g2[u] = El<kF16>::kNegInf2;
    zm = kTopkFloor;
    s = 0.f;
    auto add4 = [&](const uint4 (&q)[4], uint32_t m2) {
        const float2 mf = El<kF16>::unpack2(m2);
        const float zn = fmaxf(zm, fmaxf(mf.x, mf.y));
        float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 x = __fmul2_rn(__fadd2_rn(El<kF16>::unpack2(w[k]), splat2(-zn)), splat2(scale));
                acc[k & 1] = __fadd2_rn(acc[k & 1], make_float2(ex2(x.x), ex2(x.y)));
            }
        }
        s = fmaf(s, ex2((zm - zn) * scale), (acc[0].x + acc[0].y) + (acc[1].x + acc[1].y));
        zm = zn;
    };
    const uint4 none = make_uint4(El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2);
    auto vec_max = [&](const uint4& q) { return max2<kF16>(max2<kF16>(q.x, q.y), max2<kF16>(q.z, q.w)); };
    const uint32_t last = r.nvec - 1;           // vectors 1 .. last-1 lie inside the row
    uint32_t v0 = 1 + tid;
    for (; v0 + (kTopkGroups - 1) * NT < last; v0 += kTopkGroups * NT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint4 q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u] = load_streaming(r.vecs + v0 + (4 * h + u) * NT);
            uint32_t vm[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                vm[u] = vec_max(q[u]);
                g2[4 * h + u] = max2<kF16>(g2[4 * h + u], vm[u]);
            }
            add4(q, max2<kF16>(max2<kF16>(vm[0], vm[1]), max2<kF16>(vm[2], vm[3])));
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {               // the rest: fewer than eight vectors
        if (v0 + 4 * h * NT < last) {
            uint4 q[4];
            uint32_t m2 = El<kF16>::kNegInf2;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t v = v0 + (4 * h + u) * NT;
                q[u] = none;
                if (v < last) q[u] = load_streaming(r.vecs + v);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t vm = vec_max(q[u]);
                g2[4 * h + u] = max2<kF16>(g2[4 * h + u], vm);
                m2 = max2<kF16>(m2, vm);
            }
            add4(q, m2);
        }
    }
    if (tid == 0 || (tid == NT - 1 && last > 0)) {
        const uint4 q[4] = {span_vec<kF16>(r, tid == 0 ? 0u : last), none, none, none};
        add4(q, vec_max(q[0]));
    }
}

// ---------------------------------------------------------------- a row per block
// A thread's groups are eight: its vectors j with equal j mod 8.  Rows with more candidates than the list holds (long runs
// of equal values, rows sorted against the groups) are selected by bisection over the 16-bit values with repeated reads of
// the row.
// NT threads per row; as many blocks per SM as registers allow, so that some stream while others select.
// What the threads of a row share.
template <int NT>
struct TopkShared {
    unsigned long long cand[kTopkCandidates];
    uint16_t group[kTopkGroups * NT];
    uint32_t scratch[2 * (NT / 32)];
    float2 part[NT / 32];
    uint32_t lo[NT / 32], hi[NT / 32];
    uint32_t n[2];                      // qualifying groups, candidates: zero when a selection starts
};

// Selects the K best entries of a row from what its NT threads saw of it, and writes them.
template <int NT, bool kF16>
__device__ __forceinline__ void select_row(const TopkArgs& p, const RowSpan& r, TopkShared<NT>& sh, int tid,
                                           const uint32_t (&g2)[kTopkGroups], float zm, float s, int& turn, int* ids, float* lps)
{
    constexpr int kWarps = NT / 32;
    const int warp = tid >> 5, lane = tid & 31;
    const uint32_t empty = key_of_neg_inf<kF16>();
    const uint32_t last = r.nvec - 1;                              // vectors 1 .. last-1 belong to groups
    // ---- block totals: the row's maximum and sum; smallest and largest of the threads' maxima
    uint32_t key[kTopkGroups], top = 0u;
#pragma unroll
    for (int u = 0; u < kTopkGroups; ++u) {
        key[u] = max(order_key(g2[u] & 0xffffu), order_key(g2[u] >> 16));
        if (key[u] <= empty) key[u] = 0;                       // nothing in it to select
        top = max(top, key[u]);
    }
    float zw = zm;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) zw = fmaxf(zw, __shfl_xor_sync(0xffffffffu, zw, o));
    float sw = s * ex2((zm - zw) * p.scale);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sw += __shfl_xor_sync(0xffffffffu, sw, o);
    uint32_t lo = __reduce_min_sync(0xffffffffu, top), hi = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) { sh.part[warp] = make_float2(zw, sw); sh.lo[warp] = lo; sh.hi[warp] = hi; }
    row_sync<NT>();
    float zt = kTopkFloor, st = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) { zt = fmaxf(zt, sh.part[w].x); lo = min(lo, sh.lo[w]); hi = max(hi, sh.hi[w]); }
#pragma unroll
    for (int w = 0; w < kWarps; ++w) st += sh.part[w].y * ex2((sh.part[w].x - zt) * p.scale);
    const float l2 = log2f(st);

    // ---- a bound that K groups reach
    uint32_t end = hi + 1u;                                    // nothing reaches this
    if (p.K <= NT / 2) {
        // the K-th largest of the threads' maxima, by bisection: a thread's eight groups count as one, which costs a
        // few more candidates (74 instead of 65 for K = 64 of 256) and an eighth of the comparisons
        lo = max(lo, empty + 1u);
        if (row_count<NT>(top >= lo) < p.K) lo = end = empty + 1u;   // fewer threads with an entry than K
        while (end > lo + 1u) {
            const uint32_t mid = (lo + end) >> 1;
            if (row_count<NT>(top >= mid) >= p.K) lo = mid; else end = mid;
        }
    } else {
        // the K-th largest of all group maxima, by trisection (two counts of at most 2^13 in one reduction)
        lo = empty + 1u;
        uint32_t n = 0;
#pragma unroll
        for (int u = 0; u < kTopkGroups; ++u) n += key[u] >= lo ? 1u : 0u;
        if (block_sum<NT>(n, sh.scratch, turn) < (uint32_t)p.K) end = lo;
        while (end > lo + 1u) {
            const uint32_t d = end - lo, p1 = lo + max(1u, d / 3u), p2 = max(p1, lo + 2u * d / 3u);
            n = 0;
#pragma unroll
            for (int u = 0; u < kTopkGroups; ++u) n += (key[u] >= p1 ? 1u : 0u) + (key[u] >= p2 ? 65536u : 0u);
            n = block_sum<NT>(n, sh.scratch, turn);
            if ((n >> 16) >= (uint32_t)p.K) lo = p2;
            else if ((n & 0xffffu) >= (uint32_t)p.K) { lo = p1; end = p2; }      // p1 < p2 here: their counts differ
            else end = p1;
        }
    }

    // ---- the groups that reach it, and their entries that do; the two outer vectors always
    {
        uint32_t mine = 0;
#pragma unroll
        for (int u = 0; u < kTopkGroups; ++u) mine += key[u] >= lo ? 1u : 0u;
        uint32_t at = mine ? atomicAdd(&sh.n[0], mine) : 0u;
#pragma unroll
        for (int u = 0; u < kTopkGroups; ++u)
            if (key[u] >= lo) sh.group[at++] = (uint16_t)(u * NT + tid);
    }
    if (tid == 0 || (tid == NT - 1 && last > 0)) collect_vec<kF16>(r, tid == 0 ? 0u : last, lo, sh.cand, &sh.n[1]);
    row_sync<NT>();
    // (a group's vectors are dealt to a power of two of neighbouring threads)
    const uint32_t rounds = max(1u, (last + kTopkGroups * NT - 1) / (kTopkGroups * NT)), log_rounds = 32 - __clz((int)(rounds - 1));
    const uint32_t items = sh.n[0] << log_rounds;
    for (uint32_t it = tid; it < items; it += 2 * NT) {
        uint32_t v[2];
        uint4 q[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {                          // both in flight
            const uint32_t x = it + h * NT;
            v[h] = last;
            if (x < items) v[h] = 1u + sh.group[x >> log_rounds] + (x & ((1u << log_rounds) - 1u)) * (kTopkGroups * NT);
            if (v[h] < last) q[h] = load_streaming(r.vecs + v[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (v[h] < last) collect_entries<kF16>(r, q[h], v[h], lo, sh.cand, &sh.n[1]);
    }
    row_sync<NT>();
    uint32_t n = sh.n[1];
    if (n > (uint32_t)kTopkCandidates) n = topk_bisect<NT, kF16>(r, (uint32_t)p.K, sh.cand, &sh.n[1], sh.scratch, turn);

    // ---- ranks: the number of larger candidates
    for (uint32_t c = tid; c < n; c += NT) {
        const unsigned long long mine = sh.cand[c];
        uint32_t rank = 0;
#pragma unroll 4
        for (uint32_t o = 0; o < n; ++o) rank += sh.cand[o] > mine ? 1u : 0u;
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

constexpr int topk_blocks_per_sm(int threads) { return threads >= 1024 ? 1 : 1024 / threads; }

template <int NT, bool kF16>
__global__ void __launch_bounds__(NT, topk_blocks_per_sm(NT)) topk_block_kernel(TopkArgs p)
{
    __shared__ TopkShared<NT> sh;
    __shared__ long long s_row[2];
    __shared__ long long s_cnt[33];
    const int tid = threadIdx.x;
    int turn = 0;

    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const long long total = (long long)p.B * p.T;
    const bool one_each = (long long)gridDim.x >= total;   // no counter: block i has row i
    if (tid == 0) s_row[0] = one_each ? (long long)blockIdx.x : (long long)atomicAdd(p.row_counter, 1u);

    for (int i = 0;; ++i) {
        __syncthreads();                            // s_row[i & 1] is there; the previous row's shared data has been read
        const long long row = s_row[i & 1];
        if (row >= total) break;
        if (tid == 0) {
            s_row[(i + 1) & 1] = one_each ? total : (long long)atomicAdd(p.row_counter, 1u);   // the next row, in flight during this one
            sh.n[0] = sh.n[1] = 0;
        }
        const int b = (int)(row / p.T), t = (int)(row % p.T);
        int* ids = p.ids + row * p.K;
        float* lps = p.logprobs + row * p.K;
        if (t >= clamp_len(__ldg(p.lengths + b), p.T)) {
            for (int k = tid; k < p.K; k += NT) { ids[k] = 0; lps[k] = 0.f; }
            continue;
        }
        const RowSpan r = row_span(p.logits + (long long)b * p.stride_b + (long long)t * p.stride_t, p.V);

        // ---- the stream
        uint32_t g2[kTopkGroups];
        float zm, s;
        stream_row<NT, kF16>(r, tid, p.scale, g2, zm, s);

        select_row<NT, kF16>(p, r, sh, tid, g2, zm, s, turn, ids, lps);
    }
    if (blockIdx.x == 0) block_count_valid(p.lengths, p.B, p.T, s_cnt, p.status);   // flags lengths out of range
    if (tid == 0 && !one_each) {
        if (atomicAdd(p.ticket, 1u) == gridDim.x - 1) { *p.ticket = 0u; *p.row_counter = 0u; }
    }
}

// ---------------------------------------------------------------- log-probs of few rows
// The log-prob of the generated token for batches that do not fill the device with a row per warp (logprob_warp_kernel): a
// row per block, streamed as above, all of a row's loads in flight at once.  64 rows of 32000: 7 us against 20 us.
struct BlockLpArgs {
    const uint16_t* logits;
    long long stride_b, stride_t;
    const long long* ids;
    long long ids_stride_b;
    const int* lengths;
    int B, T, V;
    float* out_lp;
    unsigned* status;
};

template <int NT, bool kF16>
__global__ void __launch_bounds__(NT, 1024 / NT) logprob_block_kernel(BlockLpArgs p)
{
    __shared__ float2 s_part[2][NT / 32];
    __shared__ long long s_cnt[33];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const long long total = (long long)p.B * p.T;
    int par = 0;                                                     // set of parts of the next valid row
    for (long long row = blockIdx.x; row < total; row += gridDim.x) {
        const int b = (int)(row / p.T), t = (int)(row % p.T);
        if (t >= clamp_len(__ldg(p.lengths + b), p.T)) {
            if (tid == 0) p.out_lp[row] = 0.f;
            continue;
        }
        const uint16_t* z16 = p.logits + (long long)b * p.stride_b + (long long)t * p.stride_t;
        float zy = 0.f;
        bool bad_id = false;
        if (tid == 0) {                                              // in flight during the stream
            const long long y = __ldg(p.ids + (long long)b * p.ids_stride_b + t);
            bad_id = y < 0 || y >= p.V;
            if (bad_id) atomicOr(p.status, kErrIdRange);
            else zy = El<kF16>::widen(__ldg(z16 + y));
        }
        uint32_t g2[kTopkGroups];
        float zm, s;
        stream_row<NT, kF16>(row_span(z16, p.V), tid, kLog2e, g2, zm, s);
        float zw = zm;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) zw = fmaxf(zw, __shfl_xor_sync(0xffffffffu, zw, o));
        float sw = s * ex2((zm - zw) * kLog2e);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sw += __shfl_xor_sync(0xffffffffu, sw, o);
        if (lane == 0) s_part[par][warp] = make_float2(zw, sw);
        // The two sets of parts alternate from one valid row to the next: a set is written again behind the barrier of the row
        // between, which thread 0 reaches when it has read the set.  (A padded row passes no barrier and takes no set.)
        __syncthreads();
        if (tid == 0) {
            float zt = kTopkFloor, st = 0.f;
            for (int w = 0; w < NT / 32; ++w) zt = fmaxf(zt, s_part[par][w].x);
            for (int w = 0; w < NT / 32; ++w) st += s_part[par][w].y * ex2((s_part[par][w].x - zt) * kLog2e);
            // (the difference of the logits is exact; through kLog2e, 1.3e-8 below log2(e), every log-prob of a sequence would
            // be 7e-8 too large)
            p.out_lp[row] = bad_id ? 0.f : (float)((double)zy - (double)zt - 0.6931471805599453 * log2_split(st));
        }
        par ^= 1;
    }
    if (blockIdx.x == 0) block_count_valid(p.lengths, p.B, p.T, s_cnt, p.status);   // flags lengths out of range
}

}  // namespace rlhf
