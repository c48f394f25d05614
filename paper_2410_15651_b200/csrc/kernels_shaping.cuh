// Shaped logits: the distribution that a rollout's tokens are drawn from, and log-probs and gradients under it.
//
// Row (b,t) of the logits is shaped by what stands before it.  With H the prompt's tokens and those of the answer before
// row t, and c_v how often the answer has v so far,
//     x_v = ((pen(z_v) - f c_v - p [c_v > 0]) + bias_v) / tau    where the mask allows v, else -inf,
//     pen(z) = z r for z < 0 and z / r for others, where v is in H; z elsewhere.
// One kernel streams the rows in five modes: x itself in 16 or 32 bits, the gradient through it, log-probs of the generated
// tokens under softmax(x), and the gradient of those.
//
// What bounds it: HBM, if the history costs nothing per row.  A block therefore keeps one slice of one sequence's vocabulary
// (up to 16384 entries) and walks down the rows of a segment: a bit per entry says "in H" and an integer holds c_v, both in
// shared memory, built once per segment from the token lists (integer atomics: any order gives the same table) and then
// moved from row to row by one token.  A vector of eight entries whose byte of bits is 0, which is most of them, pays one
// byte load from shared memory.
#pragma once
#include "common.cuh"

namespace rlhf {

constexpr unsigned kErrValueRange = 128u;

constexpr int kShapeThreads = 512;
constexpr int kShapeMaxRows = 32;           // rows of a segment
constexpr int kShapeMaxCluster = 8;
constexpr int kShapeSliceVecs = 2048;       // vectors of eight entries per block

enum : int { kShape16 = 0, kShape32 = 1, kShapeBwd = 2, kShapeLp = 3, kShapeLpBwd = 4 };

struct ShapingArgs {
    const long long* tokens;                // [b*tokens_stride_b + i], i < S
    long long tokens_stride_b;
    int S;
    const int* start;                       // tokens before a sequence's first row; null: 0
    const long long* prompt;
    long long prompt_stride_b;
    const int* prompt_lengths;              // null: P
    int P;
    const float* repetition;                // [B] each; null: neutral
    const float* frequency;
    const float* presence;
    const float* temperature;
    const float* bias;
    long long bias_stride_b;
    const uint32_t* mask;                   // bit v % 32 of word v / 32
    long long mask_stride_b, mask_stride_t;
};

struct ShapeKernelArgs {
    ShapingArgs sh;
    const uint16_t* src;                    // logits; kShapeBwd: the gradient with respect to the shaped logits
    long long src_stride_b, src_stride_t;
    const uint16_t* logits;                 // kShapeBwd only
    long long logits_stride_b, logits_stride_t;
    void* dst;                              // rows written (not kShapeLp)
    long long dst_stride_b, dst_stride_t;
    const int* lengths;
    int B, T, V;
    const long long* ids;                   // kShapeLp, kShapeLpBwd
    long long ids_stride_b;
    float* out_lp;                          // kShapeLp
    float* out_lse;                         // [B,T,2]
    float* out_entropy;                     // or null
    const float* lp;                        // kShapeLpBwd
    const float* lse;
    const float* entropy;
    const float* grad_lp;
    const float* grad_entropy;              // or null
    unsigned* status;
    int rows_per_item;
    int n_slices;                           // slices of a row
    int cluster;                            // blocks that share an item's slices
    int slice_vecs;
    int bits_words;                         // words of the bit table in shared memory
    int uses_history, uses_counts;
    int sparse;                             // in place and nothing but penalties: only entries of H are touched
};

// What a thread needs of a row while it streams it.
struct ShapeRow {
    const uint16_t* src;
    const uint32_t* mask;
    int oo;                                 // entries of the first vector that precede the row
    int delta;                              // entries by which the source is off the vectors' boundaries
    int end;                                // one past the block's last vector
    // kShapeLpBwd
    float hi, lo, lp, g, h, ent;
    int y;
};

__device__ __forceinline__ float warp_max(float v)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ uint4 load_stream(const void* p)
{
    return __ldcs((const uint4*)p);
}

// Entries delta .. delta+7 of the sixteen in lo, hi.
__device__ __forceinline__ uint4 shift_entries(const uint4& lo, const uint4& hi, int delta)
{
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (delta & 4) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (delta & 2) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 1];
    }
    if (delta & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <bool kF16>
__device__ __forceinline__ void widen8(const uint4& q, float (&z)[8])
{
    const float2 a = El<kF16>::unpack2(q.x), b = El<kF16>::unpack2(q.y), c = El<kF16>::unpack2(q.z), d = El<kF16>::unpack2(q.w);
    z[0] = a.x; z[1] = a.y; z[2] = b.x; z[3] = b.y; z[4] = c.x; z[5] = c.y; z[6] = d.x; z[7] = d.y;
}

// Entries of one row's partial sums: sum of exp(x - m), and of exp(x - m) (x - m) for the entropy.
struct LpAcc {
    float m, s, ez;
};

constexpr float kLpClamp = -104.f;          // exp of it is 0 in fp32: makes -inf a finite factor of 0

__device__ __forceinline__ LpAcc lp_merge(const LpAcc& a, const LpAcc& b)
{
    const float m = fmaxf(a.m, b.m);
    const float da = m - a.m, db = m - b.m, ca = ex2(-da * kLog2e), cb = ex2(-db * kLog2e);
    LpAcc r;
    r.m = m;
    r.s = a.s * ca + b.s * cb;
    // (an empty partial sum has s = ez = 0 and da up to 1e38: its product stays 0)
    r.ez = ca * (a.ez - da * a.s) + cb * (b.ez - db * b.s);
    return r;
}

// kAny: rows of any alignment.  The vectors then follow the rows that are written (the source's where none are), and a source
// that is off them by `delta` entries is shifted into place from two aligned loads.
template <int kMode, bool kF16, bool kAny>
__global__ void __launch_bounds__(kShapeThreads, 2) shaping_kernel(const __grid_constant__ ShapeKernelArgs a)
{
    constexpr bool kLp = kMode == kShapeLp, kLpBwd = kMode == kShapeLpBwd, kBwd = kMode == kShapeBwd, k32 = kMode == kShape32;
    constexpr int U = kAny ? 2 : 4;                        // vectors of a thread in flight
    constexpr int kWarps = kShapeThreads / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* s_bits = (uint32_t*)smem;
    int* s_cnt = (int*)(smem + 4 * (size_t)a.bits_words);
    __shared__ LpAcc s_part[kLp ? kShapeMaxRows : 1][kLp ? kWarps : 1];
    __shared__ float4 s_row[kLp ? kShapeMaxRows : 1];      // the block's sums of a row (m, s, ez) and x of the generated token
    __shared__ float s_zy[kLp ? kShapeMaxRows : 1];

    const ShapingArgs& sh = a.sh;
    const int tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, lane = tid & 31;
    const int C = a.cluster;
    const int rank = (int)(blockIdx.x % (unsigned)C);
    const int item = (int)(blockIdx.x / (unsigned)C);
    const int b = item % a.B, t0 = item / a.B * a.rows_per_item;
    const int t1 = min(a.T, t0 + a.rows_per_item);
    const int V = a.V, SV = a.slice_vecs;
    const int n_ent = SV * 8 + (kAny ? 16 : 0);

    auto clear_table = [&]() {
        if (!a.uses_history) return;
        for (int i = tid; i < a.bits_words; i += nt) s_bits[i] = 0u;
        if (a.uses_counts) {
            int4* c4 = (int4*)s_cnt;
            for (int i = tid; i < n_ent / 4; i += nt) c4[i] = make_int4(0, 0, 0, 0);
        }
    };
    clear_table();

    pdl_wait_prior_grid();                                 // nothing above touches global memory
    pdl_release_next_grid();

    const int len_in = __ldg(a.lengths + b);
    const int len = clamp_len(len_in, a.T);
    const int tv = min(t1, len);                           // the segment's valid rows are t0 .. tv-1
    const bool reports = rank == 0 && tid == 0 && t0 == 0;
    if (reports && len_in != len) atomicOr(a.status, kErrLengthRange);

    int first = sh.start ? __ldg(sh.start + b) : 0;
    int plen = sh.P;
    if (sh.prompt_lengths) plen = __ldg(sh.prompt_lengths + b);
    if (reports && (first < 0 || (sh.tokens && len > 0 && (long long)first + len - 1 > sh.S) || plen < 0 || plen > sh.P))
        atomicOr(a.status, kErrLengthRange);
    first = max(first, 0);
    plen = clamp_len(plen, sh.P);

    // the sequence's settings; one that is out of range is neutral
    float rep = 1.f, freq = 0.f, pres = 0.f, tau = 1.f;
    bool bad = false;
    if (sh.repetition) { rep = __ldg(sh.repetition + b); if (!(rep >= 1e-3f && rep <= 1e18f)) { rep = 1.f; bad = true; } }
    if (sh.frequency) { freq = __ldg(sh.frequency + b); if (!(fabsf(freq) <= 1e18f)) { freq = 0.f; bad = true; } }
    if (sh.presence) { pres = __ldg(sh.presence + b); if (!(fabsf(pres) <= 1e18f)) { pres = 0.f; bad = true; } }
    if (sh.temperature) { tau = __ldg(sh.temperature + b); if (!(tau >= 1e-3f && tau <= 1e18f)) { tau = 1.f; bad = true; } }
    if (reports && bad) atomicOr(a.status, kErrValueRange);
    const float inv_rep = 1.f / rep, inv_tau = 1.f / tau;
    const float* bias = sh.bias ? sh.bias + (long long)b * sh.bias_stride_b : nullptr;
    const int mask_words = (V + 31) >> 5;

    auto dst_row = [&](int t) {
        const long long at = (long long)b * a.dst_stride_b + (long long)t * a.dst_stride_t;
        return k32 ? (void*)((float*)a.dst + at) : (void*)((uint16_t*)a.dst + at);
    };
    auto offset_of = [&](int t) {                          // ShapeRow::oo
        if (!kAny) return 0;
        if (kLp) return (int)(((uintptr_t)(a.src + (long long)b * a.src_stride_b + (long long)t * a.src_stride_t) >> 1) & 7);
        return k32 ? (int)(((uintptr_t)dst_row(t) >> 2) & 3) : (int)(((uintptr_t)dst_row(t) >> 1) & 7);
    };

    const int n_sub = kLp ? (a.n_slices + C - 1) / C : 1;
    for (int sub = 0; sub < n_sub; ++sub) {
        const int slice = sub * C + rank;
        const int begin = slice * SV;
        const int tb = begin * 8 - (kAny ? 8 : 0);         // entry of the table's first bit
        if (sub > 0) {
            __syncthreads();
            clear_table();
        }

        auto row_at = [&](int t) {
            ShapeRow r;
            r.src = a.src + (long long)b * a.src_stride_b + (long long)t * a.src_stride_t;
            r.mask = sh.mask ? sh.mask + (long long)b * sh.mask_stride_b + (long long)t * sh.mask_stride_t : nullptr;
            r.oo = offset_of(t);
            r.delta = kAny ? ((int)((uintptr_t)r.src >> 1) - r.oo) & 7 : 0;
            r.end = min(begin + SV, (r.oo + V + 7) >> 3);
            if (kLp || kLpBwd) {
                const long long y = __ldg(a.ids + (long long)b * a.ids_stride_b + t);
                r.y = y < 0 || y >= V ? -1 : (int)y;
            }
            if (kLpBwd) {
                const long long flat = (long long)b * a.T + t;
                const float2 n = __ldg((const float2*)a.lse + flat);
                r.hi = n.x;
                r.lo = n.y;
                r.lp = __ldg(a.lp + flat);
                r.g = r.y >= 0 ? __ldg(a.grad_lp + flat) : 0.f;
                r.h = r.ent = 0.f;
                if (a.grad_entropy) {
                    r.h = __ldg(a.grad_entropy + flat);
                    r.ent = __ldg(a.entropy + flat);
                }
            }
            return r;
        };

        struct Vec { uint4 lo, hi; uint32_t m0, m1; };     // (hi and m1 are used with kAny only)
        auto load = [&](const ShapeRow& r, int i) {
            Vec v{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0), ~0u, ~0u};
            if (i >= r.end) return v;
            if (!kAny) {
                v.lo = load_stream((const uint4*)r.src + i);
                if (r.mask) v.m0 = __ldg((const uint8_t*)r.mask + i);
            } else {
                const int e = 8 * i - r.oo, s = e - r.delta;           // s: first entry of the aligned load
                if (s + 8 > 0 && s < V) v.lo = load_stream(r.src + s);
                if (r.delta && s + 16 > 0 && s + 8 < V) v.hi = load_stream(r.src + s + 8);
                if (r.mask) {
                    const int w = e >> 5;
                    v.m0 = w >= 0 ? __ldg(r.mask + w) : 0u;
                    v.m1 = w + 1 < mask_words ? __ldg(r.mask + w + 1) : 0u;
                }
            }
            return v;
        };
        auto bits_of = [&](int i, int oo) -> uint32_t {
            if (!a.uses_history) return 0u;
            if (!kAny) return ((const uint8_t*)s_bits)[i - begin];
            const int el = 8 * i - oo - tb;
            return __funnelshift_r(s_bits[el >> 5], s_bits[(el >> 5) + 1], el & 31) & 0xffu;
        };

        // Whether the entry is the block's; marks it.
        auto in_table = [&](long long v) { return v >= max(tb, 0) && v < (long long)tb + n_ent && v < V; };
        auto mark = [&](int v, bool answer) {
            const int el = v - tb;
            atomicOr(s_bits + (el >> 5), 1u << (el & 31));
            if (answer && a.uses_counts) atomicAdd(s_cnt + el, 1);
        };

        ShapeRow row{};
        Vec q[U], nq[U];
        if (t0 < tv && !a.sparse) {                        // in flight while the table is built
            row = row_at(t0);
#pragma unroll
            for (int u = 0; u < U; ++u) q[u] = load(row, begin + u * nt + tid);
        }

        if (a.uses_history && t0 < tv) {
            __syncthreads();
            bool bad_id = false;
            const long long* p = sh.prompt + (long long)b * sh.prompt_stride_b;
            for (int i = tid; i < plen; i += nt) {
                const long long v = __ldg(p + i);
                if (in_table(v)) mark((int)v, false);
                else if (v < -1 || v >= V) bad_id = true;
            }
            const long long* k = sh.tokens + (long long)b * sh.tokens_stride_b;
            const int n = sh.tokens ? (int)min((long long)first + t0, (long long)sh.S) : 0;
            for (int i = tid; i < n; i += nt) {
                const long long v = __ldg(k + i);
                if (in_table(v)) mark((int)v, true);
                else if (v < -1 || v >= V) bad_id = true;
            }
            if (bad_id) atomicOr(a.status, kErrIdRange);
            __syncthreads();
        }

        // ---- one vector: entries e .. e+7 in x, shaped
        auto shape8 = [&](float (&x)[8], uint32_t bits, int e, uint32_t allowed) -> uint32_t {
            uint32_t neg = 0;                              // entries of H whose logit is negative
            if (bits) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (bits >> j & 1u) {
                        const bool n = x[j] < 0.f;
                        neg |= (n ? 1u : 0u) << j;
                        x[j] *= n ? rep : inv_rep;
                        if (a.uses_counts) {
                            const int c = s_cnt[e + j - tb];
                            if (c > 0) x[j] = fmaf(-freq, (float)c, x[j]) - pres;
                        }
                    }
            }
            if (bias) {
                if (e >= 0 && e + 8 <= V && ((uintptr_t)(bias + e) & 15) == 0) {
                    const float4 u = __ldg((const float4*)(bias + e)), w = __ldg((const float4*)(bias + e) + 1);
                    x[0] += u.x; x[1] += u.y; x[2] += u.z; x[3] += u.w;
                    x[4] += w.x; x[5] += w.y; x[6] += w.z; x[7] += w.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (e + j >= 0 && e + j < V) x[j] += __ldg(bias + e + j);
                }
            }
            if (sh.temperature) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= inv_tau;
            }
            if (sh.mask) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = allowed >> j & 1u ? x[j] : -INFINITY;
            }
            return neg;
        };
        // ---- the gradient of eight entries, from the one with respect to x
        auto through8 = [&](float (&d)[8], uint32_t bits, uint32_t neg, uint32_t allowed) {
            if (sh.temperature) {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] *= inv_tau;
            }
            if (bits && sh.repetition) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (bits >> j & 1u) d[j] *= neg >> j & 1u ? rep : inv_rep;
            }
            if (sh.mask) {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = allowed >> j & 1u ? d[j] : 0.f;
            }
        };
        auto store8 = [&](void* dst, int e, const float (&x)[8]) {
            if (k32) {
                float* o = (float*)dst + e;
                if (e >= 0 && e + 8 <= V) {
                    __stcs((float4*)o, make_float4(x[0], x[1], x[2], x[3]));
                    __stcs((float4*)o + 1, make_float4(x[4], x[5], x[6], x[7]));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (e + j >= 0 && e + j < V) o[j] = x[j];
                }
                return;
            }
            uint16_t* o = (uint16_t*)dst + e;
            const uint4 w = make_uint4(El<kF16>::pack2(x[0], x[1]), El<kF16>::pack2(x[2], x[3]), El<kF16>::pack2(x[4], x[5]),
                                       El<kF16>::pack2(x[6], x[7]));
            if (e >= 0 && e + 8 <= V) {
                __stcs((uint4*)o, w);
            } else {
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e + j >= 0 && e + j < V) o[j] = (uint16_t)(ww[j >> 1] >> (16 * (j & 1)));
            }
        };

        LpAcc acc{kFloorM, 0.f, 0.f};
        const bool want_ent = kLp && a.out_entropy != nullptr;
        auto lp_add = [&](const float (&x)[8]) {
            float d[8], e[8], vs, vz = 0.f;
            auto sums = [&]() {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = x[j] - acc.m;
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = ex2(d[j] * kLog2e);
                vs = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            };
            sums();
            if (!(vs <= 1.8446744e19f)) {
                // a first vector, or one more than 64 binades above the reference
                float m = kFloorM;
#pragma unroll
                for (int j = 0; j < 8; ++j) m = fmaxf(m, x[j]);
                const float up = m - acc.m, sc = ex2(-up * kLog2e);
                acc.ez = sc * (acc.ez - up * acc.s);
                acc.s *= sc;
                acc.m = m;
                sums();
            }
            acc.s += vs;
            if (want_ent) {
#pragma unroll
                for (int j = 0; j < 8; ++j) vz = fmaf(e[j], fmaxf(d[j], kLpClamp), vz);
                acc.ez += vz;
            }
        };

        auto process = [&](const Vec& v, int i, int t) {
            if (i >= row.end) return;
            const int e = 8 * i - row.oo;
            const uint32_t bits = bits_of(i, row.oo);
            uint32_t allowed = v.m0;
            if (kAny && sh.mask) allowed = __funnelshift_r(v.m0, v.m1, e & 31);
            const uint4 w = kAny ? shift_entries(v.lo, v.hi, row.delta) : v.lo;
            float x[8];
            widen8<kF16>(w, x);
            if (kBwd) {
                uint32_t neg = 0;
                if (bits && sh.repetition) {
                    const uint16_t* z = a.logits + (long long)b * a.logits_stride_b + (long long)t * a.logits_stride_t;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (bits >> j & 1u) neg |= (El<kF16>::widen(__ldg(z + e + j)) < 0.f ? 1u : 0u) << j;
                }
                through8(x, bits, neg, allowed);
                store8(dst_row(t), e, x);
                return;
            }
            const uint32_t neg = shape8(x, bits, e, allowed);
            if (kMode == kShape16 || k32) {
                store8(dst_row(t), e, x);
                return;
            }
            if (kLp) {
                if (e < 0 || e + 8 > V) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (e + j < 0 || e + j >= V) x[j] = -INFINITY;
                }
                const int yj = row.y - e;
                if (yj >= 0 && yj < 8 && row.y >= 0) {
                    // the generated token's own term is kept apart
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j == yj) { s_zy[t - t0] = x[j]; x[j] = -INFINITY; }
                }
                lp_add(x);
            } else {
                // dx_v = g ([v == y] - p_v) - h p_v (log p_v + H)
                const float nlo = row.lo == -INFINITY ? 0.f : -row.lo;         // (a row that is all -inf has p = 0)
                float d[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float lq = (x[j] - row.hi) + nlo;
                    const float p = ex2(lq * kLog2e);
                    d[j] = -row.g * p;
                    if (a.grad_entropy) d[j] = fmaf(-row.h * p, fmaxf(lq, kLpClamp) + row.ent, d[j]);
                }
                const int yj = row.y - e;
                if (yj >= 0 && yj < 8 && row.y >= 0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j == yj) {
                            // 1 - p without cancellation
                            const float own = -row.g * expm1f(row.lp);
                            const float lq = (x[j] - row.hi) + nlo;
                            d[j] = x[j] == -INFINITY ? 0.f
                                 : a.grad_entropy ? fmaf(-row.h * ex2(lq * kLog2e), lq + row.ent, own) : own;
                        }
                }
                through8(d, bits, neg, allowed);
                store8(dst_row(t), e, d);
            }
        };

        // ---- the rows
        if (a.sparse) {
            for (int t = t0; t < tv; ++t) {
                row = row_at(t);
                for (int i = begin + tid; i < row.end; i += nt)
                    if (bits_of(i, row.oo)) process(load(row, i), i, t);
                if (t + 1 < tv && sh.tokens && (long long)first + t < sh.S) {
                    const long long v = __ldg(sh.tokens + (long long)b * sh.tokens_stride_b + first + t);
                    if (in_table(v)) {
                        __syncthreads();
                        if (tid == 0) mark((int)v, true);
                        __syncthreads();
                    } else if (tid == 0 && (v < -1 || v >= V)) {
                        atomicOr(a.status, kErrIdRange);
                    }
                }
            }
        } else if (t0 < tv) {
            int t = t0, k = 0;
            long long token = -1;                          // the answer's token at row t
            auto token_at = [&](int tt) {
                return a.uses_history && sh.tokens && tt + 1 < tv && (long long)first + tt < sh.S
                           ? __ldg(sh.tokens + (long long)b * sh.tokens_stride_b + first + tt) : -1ll;
            };
            token = token_at(t);
            if (kLp || kLpBwd) {
                if (rank == 0 && sub == 0 && row.y < 0 && tid == 0) atomicOr(a.status, kErrIdRange);
            }
            for (;;) {
                int tn = t, kn = k + U * nt;
                ShapeRow next = row;
                if (begin + kn >= row.end) {
                    tn = t + 1;
                    kn = 0;
                    if (tn < tv) next = row_at(tn);
                }
                if (tn < tv) {
#pragma unroll
                    for (int u = 0; u < U; ++u) nq[u] = load(next, begin + kn + u * nt + tid);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) process(q[u], begin + k + u * nt + tid, t);
                if (tn != t) {
                    if (kLp) {
                        const float M = warp_max(acc.m);
                        const float up = M - acc.m, sc = ex2(-up * kLog2e);
                        float s = acc.s * sc, ez = sc * (acc.ez - up * acc.s);
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) {
                            s += __shfl_xor_sync(0xffffffffu, s, o);
                            if (want_ent) ez += __shfl_xor_sync(0xffffffffu, ez, o);
                        }
                        if (lane == 0) {
                            LpAcc& part = s_part[t - t0][warp];
                            part = sub == 0 ? LpAcc{M, s, ez} : lp_merge(part, LpAcc{M, s, ez});
                        }
                        acc = LpAcc{kFloorM, 0.f, 0.f};
                    }
                    if (in_table(token)) {                 // (the same for every thread)
                        __syncthreads();
                        if (tid == 0) mark((int)token, true);
                        __syncthreads();
                    } else if (tid == 0 && (token < -1 || token >= V)) {
                        atomicOr(a.status, kErrIdRange);
                    }
                    if (tn >= tv) break;
                    token = token_at(tn);
                    if (kLp || kLpBwd) {
                        if (rank == 0 && sub == 0 && next.y < 0 && tid == 0) atomicOr(a.status, kErrIdRange);
                    }
                }
                t = tn;
                k = kn;
                row = next;
#pragma unroll
                for (int u = 0; u < U; ++u) q[u] = nq[u];
            }
        }

        // ---- rows behind the sequence's end
        if (!kLp) {
            const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int t = max(t0, len); t < t1; ++t) {
                const int oo = offset_of(t), end = min(begin + SV, (oo + V + 7) >> 3);
                for (int i = begin + tid; i < end; i += nt) store8(dst_row(t), 8 * i - oo, zero);
            }
        }
    }

    if (kLp) {
        if (rank == 0) {
            for (int t = max(t0, len) + tid; t < t1; t += nt) {
                const long long flat = (long long)b * a.T + t;
                a.out_lp[flat] = 0.f;
                *((float2*)a.out_lse + flat) = make_float2(0.f, 0.f);
                if (a.out_entropy) a.out_entropy[flat] = 0.f;
            }
        }
        if (t0 >= tv) return;                              // (the whole cluster)
        __syncthreads();
        const int nw = nt >> 5;
        for (int r = warp; r < tv - t0; r += nw) {
            LpAcc p = lane < nw ? s_part[r][lane] : LpAcc{kFloorM, 0.f, 0.f};
#pragma unroll
            for (int o = kWarps / 2; o > 0; o >>= 1)
                p = lp_merge(p, LpAcc{__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                                      __shfl_xor_sync(0xffffffffu, p.ez, o)});
            if (lane == 0) s_row[r] = make_float4(p.m, p.s, p.ez, s_zy[r]);
        }
        __syncthreads();
        if (C > 1) {
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        }
        if (rank == 0) {
            for (int r = tid; r < tv - t0; r += nt) {
                const int t = t0 + r;
                const long long y = __ldg(a.ids + (long long)b * a.ids_stride_b + t);
                const bool known = y >= 0 && y < V;
                // the block that has seen the generated token
                const int owner = known ? (int)(((offset_of(t) + y) >> 3) / SV % C) : 0;
                float4 own = s_row[r];
                LpAcc p{own.x, own.y, own.z};
                float zy = own.w;
                for (int c = 1; c < C; ++c) {
                    uint32_t at;
                    float4 o;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                                 : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(s_row + r)), "r"(c));
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(o.x), "=f"(o.y), "=f"(o.z), "=f"(o.w) : "r"(at));
                    p = lp_merge(p, LpAcc{o.x, o.y, o.z});
                    if (c == owner) zy = o.w;
                }
                float ey = 0.f, dy = 0.f;
                if (known && zy > -INFINITY) {
                    // (a token far above the others: the reference follows)
                    if (zy - p.m > 44.f) p = lp_merge(p, LpAcc{zy, 0.f, 0.f});
                    dy = zy - p.m;
                    ey = ex2(dy * kLog2e);
                }
                const float total = p.s + ey, lo = logf(total);
                float lp = 0.f;
                if (known) {
                    if (zy == -INFINITY) lp = -INFINITY;
                    else lp = ey > p.s ? -log1pf(p.s / ey) : dy - lo;
                }
                const long long flat = (long long)b * a.T + t;
                a.out_lp[flat] = lp;
                *((float2*)a.out_lse + flat) = make_float2(p.m, lo);
                if (a.out_entropy)
                    a.out_entropy[flat] = total > 0.f ? lo - (p.ez + ey * fmaxf(dy, kLpClamp)) / total : 0.f;
            }
        }
        if (C > 1) {                                       // the others' rows have been read
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        }
    }
}

}  // namespace rlhf
