// Shaped logits: the distribution that a rollout's tokens are drawn from, and log-probs and gradients under it.
//
// Row (b,t) of the logits is shaped by what stands before it.  With H the prompt's tokens and those of the answer before
// row t, and c_v how often the answer has v so far,
//     x_v = ((pen(z_v) - f c_v - p [c_v > 0]) + bias_v) / tau    where the mask allows v, else -inf,
//     pen(z) = z r for z < 0 and z / r for others, where v is in H; z elsewhere.
// One kernel streams the rows in five modes: x itself in 16 or 32 bits, the gradient through it, log-probs of the generated
// tokens under softmax(x), and the gradient of those.
//
// What bounds it: HBM, if the history costs nothing per row.  shaping_kernel therefore keeps one slice of one sequence's
// vocabulary per block and walks down its rows; each of its warps has a segment of the slice (some 200 vectors of eight
// entries), buffers that bulk copies fill a row or more ahead, and nothing to wait for but these.  In shared memory the block has a
// bit per entry that says "in H, or will be within the coming 32 rows", the ascending list of those entries and, where
// penalties count, c_v of every entry; they are built where a block begins a sequence and brought up to date every 32 rows.  A warp
// streams its segment of a row as if no entry were in H, and then forms those that are (one or two per lane) by themselves,
// from the same buffer: it writes them over what the stream wrote, or, where a sum is wanted, the stream has left them out.  The
// generated token is formed apart in the same way.  Bits and counts come from atomics on whole numbers, so no result depends on
// their order.
//
// shaping_row_kernel is for decoding steps and other small batches, where latency counts: a block per row and slice, the vectors in
// registers, the list in the order in which its entries are found (each is a result of its own there).
#pragma once
#include <type_traits>

#include "async.cuh"
#include "common.cuh"

namespace rlhf {

constexpr unsigned kErrValueRange = 128u;

constexpr int kShapeWarps = 24;             // warps of a block of shaping_kernel, at most
constexpr int kShapeLpWarps = 20;           // the same of log-probs, which want 96 registers (16 x 512 of 128256 with masks and
                                            // entropy: 24 warps of 80 registers 696 us, 20 565 us, 16 675 us)
constexpr int kShapeSegment = 512;          // vectors of eight entries of a warp, at most
constexpr int kShapeRows = 32;              // rows between two updates of the table
constexpr int kShapeMaxCluster = 8;
constexpr int kShapeMaxBufs = 4;
constexpr int kShapeShortRows = 16;         // shorter sequences go to shaping_row_kernel
constexpr int kRowThreads = 256;            // threads of a block of shaping_row_kernel,
constexpr int kRowVecs = 4;                 // and vectors of a thread

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
    unsigned long long wait_limit_ns;
    int n_slices;                           // slices of a row
    int cluster;                            // kShapeLp: blocks that share a row's slices, else 1
    int segment;                            // vectors of a warp; a slice has one segment per warp
    int n_bufs;                             // buffers of a warp
    int direct;                             // a cluster per row, padded ones too, instead of a range of the valid rows (kShapeLp)
    int bits_words;                         // words of the bit table in shared memory
    int list_cap;                           // entries of the list
    int uses_history, uses_counts;
    int wide_counts;                        // counts of 32 instead of 16 bits
    int sparse;                             // in place and nothing but penalties: only entries of H are touched
};

// Shared memory of shaping_kernel, in this order: the warps' buffers, their mask words (two rows), their barriers, the bits, the
// list, the list's marks, the counts.
struct ShapeSmem {
    size_t bufs, words, bars, bits, list, marks, counts, total;
};
__host__ __device__ inline ShapeSmem shape_smem(const ShapeKernelArgs& a, int warps, bool any)
{
    const size_t buf = 16 * (size_t)a.segment + (any ? 32 : 0), entries = 8 * (size_t)a.segment * warps + (any ? 16 : 0);
    ShapeSmem s;
    s.bufs = 0;
    s.words = s.bufs + (a.sparse ? 0 : buf * warps * a.n_bufs);
    s.bars = s.words + (a.sh.mask ? 2 * 4 * ((size_t)a.segment / 4 + 4) * warps : 0);
    s.bars = (s.bars + 15) / 16 * 16;
    s.bits = s.bars + ((size_t)warps * a.n_bufs * 8 + 15) / 16 * 16;
    s.list = s.bits + 4 * (size_t)a.bits_words;
    s.marks = s.list + 2 * (size_t)a.list_cap;
    s.counts = s.marks + (size_t)a.list_cap;
    s.total = s.counts + (a.uses_counts ? (a.wide_counts ? 4 : 2) * entries : 0);
    return s;
}

// What a block knows of the sequence that it walks down.
struct ShapeWalk {
    const uint16_t* src;                    // row 0 of the sequence in each tensor
    const uint16_t* logits;
    void* dst;
    const uint32_t* mask;
    const float* bias;
    const long long* answer;
    const long long* ids;
    long long flat;                         // of row 0 in [B,T] arrays
    int first;                              // answer's tokens before row 0
    int ta, te;                             // the block's rows
    float rep, inv_rep, freq, pres, tau, inv_tau;
};

__device__ __forceinline__ float warp_max(float v)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
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

// Four pairs of 16-bit entries: those whose bit of `keep` is 0 replaced by the halves of `c`.  (Bit i of a nibble times
// 2^7 + 2^14 + 2^21 + 2^28 is the top bit of byte i, among others; a byte permutation then spreads the top bits.)
__device__ __forceinline__ uint4 keep_entries(const uint4& w, uint32_t keep, uint32_t c)
{
    const uint32_t lo = (keep & 15u) * 0x10204080u, hi = (keep >> 4 & 15u) * 0x10204080u;
    uint32_t m0, m1, m2, m3;
    asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(m0) : "r"(lo));
    asm("prmt.b32 %0, %1, 0, 0xbbaa;" : "=r"(m1) : "r"(lo));
    asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(m2) : "r"(hi));
    asm("prmt.b32 %0, %1, 0, 0xbbaa;" : "=r"(m3) : "r"(hi));
    return make_uint4((w.x & m0) | (c & ~m0), (w.y & m1) | (c & ~m1), (w.z & m2) | (c & ~m2), (w.w & m3) | (c & ~m3));
}

// Entries of one row's partial sums: sum of exp(x - m), and of exp(x - m) (x - m) for the entropy.
struct LpAcc {
    float m, s, ez;
};

constexpr float kLpClamp = -150.f;          // 2^ of it is 0 in fp32: makes -inf a finite factor of 0

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

// A lane's sums of a row's terms 2^y, y = fma(z, k, -c), c = k * ref rounded, k = log2(e) / tau: one operation per logit, exact but
// for its last rounding where z is near `ref`, however far from 0 both are.
struct LaneSums {
    float ref, c, s, ez;                    // ez: sum of 2^y y
};
constexpr float kNoRef = -3.0e38f;
__device__ __forceinline__ LaneSums lane_sums() { return LaneSums{kNoRef, 0.f, 0.f, 0.f}; }

// Raises the reference.
__device__ __forceinline__ void lane_rebase(LaneSums& a, float ref, float k)
{
    const float c = ref * k;
    if (a.ref == kNoRef) {
        a.s = a.ez = 0.f;
    } else {
        const float up = c - a.c, f = ex2(-up);
        a.ez = f * (a.ez - up * a.s);
        a.s *= f;
    }
    a.ref = ref;
    a.c = c;
}

// One more term.  (z = -inf adds 0.)
__device__ __forceinline__ void lane_add1(LaneSums& a, float z, float k, bool want_ent)
{
    if (z > kNoRef && (a.ref == kNoRef || fmaf(z, k, -a.c) > 64.f)) lane_rebase(a, z, k);
    const float y = a.ref == kNoRef ? z : fmaf(z, k, -a.c), e = ex2(y);       // (no reference: -inf or NaN)
    a.s += e;
    if (want_ent) a.ez = fmaf(e, fmaxf(y, kLpClamp), a.ez);
}

// Sixteen more.
__device__ __forceinline__ void lane_add16(LaneSums& a, const float2 (&z)[2][4], float k, bool want_ent)
{
    if (a.ref == kNoRef) {                                 // the first: their maximum, if there is one
        float m = kNoRef;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = fmaxf(m, fmaxf(z[u][j].x, z[u][j].y));
        if (m == kNoRef) return;
        lane_rebase(a, m, k);
    }
    for (bool again = false;; again = true) {              // (a loop: the registers of two copies would not fit)
        const float2 nc = splat2(-a.c), kk = splat2(k);
        float2 sum[2] = {splat2(0.f), splat2(0.f)}, ez[2] = {splat2(0.f), splat2(0.f)};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 y = __ffma2_rn(z[u][j], kk, nc);
                const float2 e = make_float2(ex2(y.x), ex2(y.y));
                sum[u] = __fadd2_rn(sum[u], e);
                if (want_ent) ez[u] = __ffma2_rn(e, make_float2(fmaxf(y.x, kLpClamp), fmaxf(y.y, kLpClamp)), ez[u]);
            }
        const float2 vs = __fadd2_rn(sum[0], sum[1]);
        if (again || vs.x + vs.y <= 1.8446744e19f) {
            a.s += vs.x + vs.y;
            if (want_ent) a.ez += (ez[0].x + ez[0].y) + (ez[1].x + ez[1].y);
            return;
        }
        // a term more than 64 binades above the reference: their maximum is the next one
        float m = kNoRef;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = fmaxf(m, fmaxf(z[u][j].x, z[u][j].y));
        if (m > a.ref) lane_rebase(a, m, k);               // (not for NaN)
    }
}

// The same in nats against ref / tau.  (The rounding of c is a factor of all of the lane's terms: taken back here.)
__device__ __forceinline__ LpAcc lane_done(const LaneSums& a, float k, float inv_tau)
{
    if (a.ref == kNoRef) return LpAcc{kFloorM, a.s, 0.f};
    const float r = fmaf(a.ref, k, -a.c), f = ex2(-r);
    return LpAcc{a.ref * inv_tau, a.s * f, kLn2 * f * fmaf(-r, a.s, a.ez)};
}

// Entries e .. e+7 of a bias row (0 outside [0,V)).
__device__ __forceinline__ void load_bias(const float* bias, int e, int V, float (&b)[8])
{
    const float* p = bias + e;
    if (e >= 0 && e + 8 <= V) {
        // the 16-byte blocks that hold them, shifted into place
        const int off = (int)((uintptr_t)p >> 2) & 3;
        const float4* q = (const float4*)(p - off);
        const float4 x = __ldg(q), y = __ldg(q + 1);
        float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
        if (off) z = __ldg(q + 2);
        float v[12] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
        if (off & 2) {
#pragma unroll
            for (int j = 0; j < 10; ++j) v[j] = v[j + 2];
        }
        if (off & 1) {
#pragma unroll
            for (int j = 0; j < 9; ++j) v[j] = v[j + 1];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = e + j >= 0 && e + j < V ? __ldg(p + j) : 0.f;
    }
}

// The k-th valid (or padded) row: its sequence, and how many such rows precede that sequence.  By a whole warp.
__device__ __forceinline__ void find_row(const int* __restrict__ lengths, int B, int T, bool padded, long long k, int& b, long long& before)
{
    const int lane = threadIdx.x & 31;
    before = 0;
    for (int base = 0; base < B; base += 32) {
        int n = 0;
        if (base + lane < B) {
            n = clamp_len(__ldg(lengths + base + lane), T);
            if (padded) n = T - n;
        }
        long long upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + upto > k);
        if (past) {
            const int at = __ffs(past) - 1;
            b = base + at;
            before += __shfl_sync(0xffffffffu, upto - n, at);
            return;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    b = B;
}

// Rows [t, te) of one slice become 0.
template <bool k32, bool kAny>
__device__ __forceinline__ void clear_rows(void* dst, long long stride_t, int t, int te, int begin, int SV, int V)
{
    for (; t < te; ++t) {
        char* row = (char*)dst + (k32 ? 4 : 2) * ((long long)t * stride_t);
        const int oo = kAny ? (k32 ? (int)((uintptr_t)row >> 2) & 3 : (int)((uintptr_t)row >> 1) & 7) : 0;
        const int end = min(begin + SV, (oo + V + 7) >> 3);
        for (int i = begin + (int)threadIdx.x; i < end; i += (int)blockDim.x) {
            const int e = 8 * i - oo;
            if (e >= 0 && e + 8 <= V) {
                if (k32) {
                    __stcs((float4*)((float*)row + e), make_float4(0.f, 0.f, 0.f, 0.f));
                    __stcs((float4*)((float*)row + e) + 1, make_float4(0.f, 0.f, 0.f, 0.f));
                } else {
                    __stcs((uint4*)((uint16_t*)row + e), make_uint4(0, 0, 0, 0));
                }
            } else {
                for (int j = max(0, -e); j < min(8, V - e); ++j) {
                    if (k32) ((float*)row)[e + j] = 0.f;
                    else ((uint16_t*)row)[e + j] = 0;
                }
            }
        }
    }
}

// A row's log-prob, normaliser and entropy from the sums of the C blocks of a cluster; `rows` is the calling block's, y the
// generated token (-1: unknown), which block `owner` has seen.
__device__ __forceinline__ void lp_finish(const ShapeKernelArgs& a, const float4* rows, int y, int owner, int C, long long flat)
{
    const float4 own = *rows;
    LpAcc p{own.x, own.y, own.z};
    float zy = own.w;
    for (int c = 1; c < C; ++c) {
        uint32_t at;
        float4 o;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(rows)), "r"(c));
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(o.x), "=f"(o.y), "=f"(o.z), "=f"(o.w) : "r"(at));
        p = lp_merge(p, LpAcc{o.x, o.y, o.z});
        if (c == owner) zy = o.w;
    }
    float ey = 0.f, dy = 0.f;
    if (y >= 0 && zy > -INFINITY) {
        if (zy - p.m > 44.f) p = lp_merge(p, LpAcc{zy, 0.f, 0.f});     // a token far above the others: the reference follows
        dy = zy - p.m;
        ey = ex2(dy * kLog2e);
    }
    const float total = p.s + ey, lo = logf(total);
    float lp = 0.f;
    if (y >= 0) {
        if (zy == -INFINITY) lp = -INFINITY;
        else lp = ey > p.s ? -log1pf(p.s / ey) : dy - lo;
    }
    a.out_lp[flat] = lp;
    *((float2*)a.out_lse + flat) = make_float2(p.m, lo);
    if (a.out_entropy) a.out_entropy[flat] = total > 0.f ? lo - (p.ez + (ey > 0.f ? ey * dy : 0.f)) / total : 0.f;
}

// What a row's backward pass needs (kShapeLpBwd).  With k = log2(e) / tau and the normaliser hi + lo, p = 2^(fma(z, k, -c)) q where c is
// k * (hi tau) rounded and q = exp(-lo) and that rounding; dx = p (g + h (log p + entropy)) is formed as 2^y (g + h y), with q, the
// logarithm's constant part and 1/tau in g and h.
struct ShapeNorm {
    float c, g, h;                          // of the stream
    float hi, lo, g1, h1, ent;              // of the entries that are formed by themselves: less hi and lo, less the gradients over tau
};
__device__ __forceinline__ ShapeNorm shape_norm(const ShapeKernelArgs& a, long long flat, bool known, float tau, float inv_tau)
{
    const float2 l = __ldg((const float2*)a.lse + flat);
    const float k = kLog2e * inv_tau, ref = l.x * tau;
    const float lo = l.y == -INFINITY ? 0.f : l.y;         // (a row that is all -inf has p = 0)
    ShapeNorm n;
    n.hi = -l.x;
    n.lo = -lo;
    n.g1 = known ? -__ldg(a.grad_lp + flat) * inv_tau : 0.f;
    n.h1 = a.grad_entropy ? -__ldg(a.grad_entropy + flat) * inv_tau : 0.f;
    n.ent = a.grad_entropy ? __ldg(a.entropy + flat) : 0.f;
    if (l.y == -INFINITY) {
        n.c = 3.0e38f;
        n.g = n.h = 0.f;
        return n;
    }
    n.c = ref * k;
    const float r = fmaf(ref, k, -n.c), q = expf(-lo) * ex2(-r);
    n.g = q * fmaf(n.h1, n.ent - lo - r * kLn2, n.g1);
    n.h = q * n.h1 * kLn2;
    return n;
}

// Eight entries of a row, widened and with their bias, into what is written, up to the mask.
template <int kMode>
__device__ __forceinline__ void shape8(float2 (&z)[4], float inv_tau, const ShapeNorm& n, bool with_entropy)
{
    if (kMode == kShapeLpBwd) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 y = __ffma2_rn(z[j], splat2(kLog2e * inv_tau), splat2(-n.c));
            const float2 p = make_float2(ex2(y.x), ex2(y.y));
            float2 f = splat2(n.g);
            if (with_entropy) f = __ffma2_rn(make_float2(fmaxf(y.x, kLpClamp), fmaxf(y.y, kLpClamp)), splat2(n.h), f);
            z[j] = __fmul2_rn(p, f);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = __fmul2_rn(z[j], splat2(inv_tau));
    }
}

// One entry by itself, into what is written (kShapeLp: x tau).  `raw` is the source row's entry, `by` what the penalty multiplies it by, c its
// count, `is_y` whether it is the generated token, whose log-prob is lp.
template <int kMode>
__device__ __forceinline__ float shape1(float raw, float by, uint32_t c, float freq, float pres, const float* bias, bool allowed, float inv_tau,
                                        const ShapeNorm& n, bool with_entropy, bool is_y, float lp)
{
    if (kMode == kShapeBwd) return allowed ? raw * by * inv_tau : 0.f;
    float x = raw * by;
    if (c > 0) x = fmaf(-freq, (float)c, x) - pres;
    if (bias) x += *bias;
    if (kMode == kShapeLp) return allowed ? x : -INFINITY;
    x = allowed ? x * inv_tau : -INFINITY;
    if (kMode != kShapeLpBwd) return x;
    const float lq = (x + n.hi) + n.lo, p = ex2(lq * kLog2e);
    float d = n.g1 * (is_y ? expm1f(lp) : p);              // 1 - p without cancellation
    if (with_entropy) d = fmaf(n.h1 * p, fmaxf(lq, kLpClamp) + n.ent, d);
    return x == -INFINITY ? 0.f : d * by;
}

// Writes entries e .. e+7 of a row (of [0,V)).  `ragged`: they may pass the row's ends.
template <int kMode, bool kF16>
__device__ __forceinline__ void store8(void* dst, int e, int V, bool ragged, const float2 (&z)[4], bool masked, uint32_t allowed)
{
    constexpr bool k32 = kMode == kShape32;
    constexpr uint32_t kOut2 = kMode == kShapeBwd || kMode == kShapeLpBwd ? 0u : El<kF16>::kNegInf2;       // what a masked entry gives
    const bool whole = !ragged || (e >= 0 && e + 8 <= V);
    if (k32) {
        float* o = (float*)dst + e;
        float x[8] = {z[0].x, z[0].y, z[1].x, z[1].y, z[2].x, z[2].y, z[3].x, z[3].y};
        if (masked) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = allowed >> j & 1u ? x[j] : -INFINITY;
        }
        if (whole) {
            __stcs((float4*)o, make_float4(x[0], x[1], x[2], x[3]));
            __stcs((float4*)o + 1, make_float4(x[4], x[5], x[6], x[7]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e + j >= 0 && e + j < V) o[j] = x[j];
        }
        return;
    }
    uint4 w = make_uint4(El<kF16>::pack2(z[0].x, z[0].y), El<kF16>::pack2(z[1].x, z[1].y), El<kF16>::pack2(z[2].x, z[2].y),
                         El<kF16>::pack2(z[3].x, z[3].y));
    if (masked) w = keep_entries(w, allowed, kOut2);
    uint16_t* o = (uint16_t*)dst + e;
    if (whole) {
        __stcs((uint4*)o, w);
    } else {
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (e + j >= 0 && e + j < V) o[j] = (uint16_t)(ww[j >> 1] >> (16 * (j & 1)));
    }
}
template <int kMode, bool kF16>
__device__ __forceinline__ void store1(void* dst, int v, float x)
{
    if (kMode == kShape32) ((float*)dst)[v] = x;
    else ((uint16_t*)dst)[v] = (uint16_t)El<kF16>::pack2(x, 0.f);
}

template <bool kF16>
__device__ __forceinline__ void widen8(const uint4& w, float2 (&z)[4])
{
    z[0] = El<kF16>::unpack2(w.x);
    z[1] = El<kF16>::unpack2(w.y);
    z[2] = El<kF16>::unpack2(w.z);
    z[3] = El<kF16>::unpack2(w.w);
}

__device__ __forceinline__ void add_bias8(float2 (&z)[4], const float* bias, int e, int V)
{
    float b[8];
    load_bias(bias, e, V, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = __fadd2_rn(z[j], make_float2(b[2 * j], b[2 * j + 1]));
}

// The settings of a sequence; one that is out of range is neutral.
__device__ __forceinline__ void load_settings(const ShapingArgs& sh, int b, ShapeWalk& w)
{
    float rep = sh.repetition ? __ldg(sh.repetition + b) : 1.f, tau = sh.temperature ? __ldg(sh.temperature + b) : 1.f;
    w.freq = sh.frequency ? __ldg(sh.frequency + b) : 0.f;
    w.pres = sh.presence ? __ldg(sh.presence + b) : 0.f;
    w.first = sh.start ? max(0, __ldg(sh.start + b)) : 0;
    if (!(rep >= 1e-3f && rep <= 1e18f)) rep = 1.f;
    if (!(tau >= 1e-3f && tau <= 1e18f)) tau = 1.f;
    if (!(fabsf(w.freq) <= 1e18f)) w.freq = 0.f;
    if (!(fabsf(w.pres) <= 1e18f)) w.pres = 0.f;
    w.rep = rep;
    w.inv_rep = 1.f / rep;
    w.tau = tau;
    w.inv_tau = 1.f / tau;
}

// What is wrong with the sequences' numbers, said once (by one block).
__device__ __forceinline__ void report_settings(const ShapeKernelArgs& a)
{
    const ShapingArgs& sh = a.sh;
    unsigned wrong = 0;
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const int n = __ldg(a.lengths + b);
        if (n < 0 || n > a.T) wrong |= kErrLengthRange;
        const int f = sh.start ? __ldg(sh.start + b) : 0;
        if (f < 0 || (sh.tokens && n > 0 && (long long)f + min(n, a.T) - 1 > sh.S)) wrong |= kErrLengthRange;
        if (sh.prompt_lengths && (unsigned)__ldg(sh.prompt_lengths + b) > (unsigned)sh.P) wrong |= kErrLengthRange;
        auto outside = [&](const float* p, float lo, float hi) {
            const float v = p ? __ldg(p + b) : 1.f;
            return !(v >= lo && v <= hi);
        };
        if (outside(sh.repetition, 1e-3f, 1e18f) || outside(sh.temperature, 1e-3f, 1e18f) || outside(sh.frequency, -1e18f, 1e18f) ||
            outside(sh.presence, -1e18f, 1e18f))
            wrong |= kErrValueRange;
    }
    if (wrong) atomicOr(a.status, wrong);
}

// ---------------------------------------------------------------- a block per row and slice
// Shared memory: bits, list (2 bytes; the top bit: not in H, the generated token), what the list's entries become (4 bytes), counts.
inline __host__ __device__ size_t shape_row_smem(const ShapeKernelArgs& a, bool any)
{
    const size_t entries = 8 * (size_t)a.segment + (any ? 16 : 0);
    return 4 * (size_t)a.bits_words + 6 * (size_t)a.list_cap + (a.uses_counts ? (a.wide_counts ? 4 : 2) * entries : 0);
}

template <int kMode, bool kF16, bool kAny>
__global__ void __launch_bounds__(kRowThreads, 4) shaping_row_kernel(const __grid_constant__ ShapeKernelArgs a)
{
    constexpr bool kLpBwd = kMode == kShapeLpBwd, kBwd = kMode == kShapeBwd, k32 = kMode == kShape32;
    extern __shared__ __align__(16) unsigned char smem[];
    float* const s_val = (float*)smem;
    uint32_t* const s_bits = (uint32_t*)(s_val + a.list_cap);
    uint32_t* const s_cnt = s_bits + a.bits_words;
    uint16_t* const s_list = (uint16_t*)(s_cnt + (a.uses_counts ? (8 * a.segment + (kAny ? 16 : 0)) / (a.wide_counts ? 1 : 2) : 0));
    __shared__ ShapeWalk s_w;
    __shared__ int s_n;

    const ShapingArgs& sh = a.sh;
    const int tid = threadIdx.x, V = a.V, T = a.T, SV = a.segment;
    const int n_ent = SV * 8 + (kAny ? 16 : 0);
    const unsigned flat = blockIdx.x / (unsigned)a.n_slices;
    const int slice = (int)(blockIdx.x - flat * (unsigned)a.n_slices), b = (int)(flat / (unsigned)T), t = (int)(flat - (unsigned)b * (unsigned)T);
    const int begin = slice * SV, tb = begin * 8 - (kAny ? 8 : 0);
    for (int i = tid; i < a.bits_words; i += kRowThreads) s_bits[i] = 0u;
    if (a.uses_counts)
        for (int i = tid; i < n_ent / (a.wide_counts ? 4 : 8); i += kRowThreads) ((uint4*)s_cnt)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) s_n = 0;

    pdl_wait_prior_grid();                                 // nothing above touches global memory
    pdl_release_next_grid();
    if (blockIdx.x == 0) report_settings(a);
    const uint16_t* src = a.src + (long long)b * a.src_stride_b + (long long)t * a.src_stride_t;
    const long long off = (long long)b * a.dst_stride_b + (long long)t * a.dst_stride_t;
    void* dst = k32 ? (void*)((float*)a.dst + off) : (void*)((uint16_t*)a.dst + off);
    const int oo = !kAny ? 0 : k32 ? (int)((uintptr_t)dst >> 2) & 3 : (int)((uintptr_t)dst >> 1) & 7;
    const int delta = kAny ? ((int)((uintptr_t)src >> 1) - oo) & 7 : 0;
    const int end = min(begin + SV, (oo + V + 7) >> 3);
    if (t >= __ldg(a.lengths + b)) {                       // padding
        clear_rows<k32, kAny>(dst, 0, 0, 1, begin, SV, V);
        return;
    }
    // in flight while the table is built
    uint4 q[kRowVecs], hi[kAny ? kRowVecs : 1];
    uint32_t allowed[kRowVecs];
    const uint32_t* mask = sh.mask ? sh.mask + (long long)b * sh.mask_stride_b + (long long)t * sh.mask_stride_t : nullptr;
    if (!a.sparse) {
#pragma unroll
        for (int u = 0; u < kRowVecs; ++u) {
            const int i = begin + tid + u * kRowThreads;
            allowed[u] = ~0u;
            if (i >= end) continue;
            const int e = 8 * i - oo, s = e - delta;
            if (!kAny) {
                q[u] = __ldcs((const uint4*)src + i);
                if (sh.mask) allowed[u] = __ldg((const uint8_t*)mask + i);
            } else {
                q[u] = hi[u] = make_uint4(0, 0, 0, 0);
                if (s + 8 > 0 && s < V) q[u] = __ldcs((const uint4*)(src + s));
                if (delta && s + 16 > 0 && s + 8 < V) hi[u] = __ldcs((const uint4*)(src + s + 8));
                if (sh.mask) {
                    const int w = e >> 5;
                    const uint32_t m0 = w >= 0 ? __ldg(mask + w) : 0u, m1 = w + 1 < (V + 31) >> 5 ? __ldg(mask + w + 1) : 0u;
                    allowed[u] = __funnelshift_r(m0, m1, e & 31);
                }
            }
        }
    }
    if (tid == 0) load_settings(sh, b, s_w);
    const long long lo = max(tb, 0), span = max(min((long long)tb + n_ent, (long long)V) - lo, 0ll);
    auto in_table = [&](long long v) { return (unsigned long long)v - (unsigned long long)lo < (unsigned long long)span; };
    // an entry next to the slice's border is in two tables: the block that has its vector forms it
    auto has = [&](int v) {
        const int i = (v + oo) >> 3;
        return i >= begin && i < end;
    };
    __syncthreads();
    if (a.uses_history) {
        bool bad_id = false;
        auto mark = [&](long long v, bool of_answer) {
            if (!in_table(v)) {
                if ((unsigned long long)v + 1 > (unsigned long long)V) bad_id = true;
                return;
            }
            const int el = (int)v - tb;
            const uint32_t bit = 1u << (el & 31);
            if (!(atomicOr(s_bits + (el >> 5), bit) & bit) && has((int)v)) s_list[atomicAdd(&s_n, 1)] = (uint16_t)el;
            if (of_answer && a.uses_counts) {
                if (a.wide_counts) atomicAdd(s_cnt + el, 1u);
                else atomicAdd(s_cnt + (el >> 1), 1u << (16 * (el & 1)));
            }
        };
        const int plen = sh.prompt_lengths ? clamp_len(__ldg(sh.prompt_lengths + b), sh.P) : sh.P;
        const long long* p = sh.prompt + (long long)b * sh.prompt_stride_b;
        const long long* k = sh.tokens + (long long)b * sh.tokens_stride_b;
        const int n = sh.tokens ? (int)min((long long)s_w.first + t, (long long)sh.S) : 0;
        auto scan = [&](const long long* from, int n, bool of_answer) {         // (four loads at a time: the block waits for them)
            for (int i = tid; i < n; i += 4 * kRowThreads) {
                long long v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = u * kRowThreads < n - i ? __ldg(from + i + u * kRowThreads) : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) mark(v[u], of_answer);
            }
        };
        scan(p, plen, false);
        scan(k, n, true);
        if (bad_id) atomicOr(a.status, kErrIdRange);
        __syncthreads();
    }
    int y = -1;
    ShapeNorm norm{};
    if (kLpBwd) {
        const long long id = __ldg(a.ids + (long long)b * a.ids_stride_b + t);
        const bool known = id >= 0 && id < V;
        y = known ? (int)id : -1;
        if (!known && tid == 0) atomicOr(a.status, kErrIdRange);
        norm = shape_norm(a, flat, known, s_w.tau, s_w.inv_tau);
        if (tid == 0 && known && in_table(y) && has(y) && !(a.uses_history && (s_bits[(y - tb) >> 5] >> ((y - tb) & 31) & 1u)))
            s_list[s_n++] = (uint16_t)((y - tb) | 0x8000);
        __syncthreads();
    }
    // what is formed by itself, before the row is written over (in place)
    const int n_list = s_n;
    const float inv_tau = s_w.inv_tau;
    const float* bias = sh.bias ? sh.bias + (long long)b * sh.bias_stride_b : nullptr;
    for (int k = tid; k < n_list; k += kRowThreads) {
        const int el = s_list[k] & 0x7fff, v = el + tb;
        const bool listed = !(s_list[k] & 0x8000);
        const float raw = El<kF16>::widen(src[v]);
        const float z = kBwd ? El<kF16>::widen(__ldg(a.logits + (long long)b * a.logits_stride_b + (long long)t * a.logits_stride_t + v)) : raw;
        uint32_t c = 0;
        if (a.uses_counts && listed) c = a.wide_counts ? s_cnt[el] : ((const uint16_t*)s_cnt)[el];
        const bool ok = !sh.mask || (__ldg(mask + (v >> 5)) >> (v & 31) & 1u);
        s_val[k] = shape1<kMode>(raw, listed ? (z < 0.f ? s_w.rep : s_w.inv_rep) : 1.f, c, s_w.freq, s_w.pres, bias ? bias + v : nullptr, ok, inv_tau,
                                 norm, a.grad_entropy != nullptr, v == y, kLpBwd ? __ldg(a.lp + flat) : 0.f);
    }
    if (!a.sparse) {
        // (in place: every entry that is formed by itself has been read)
        __syncthreads();
        const bool ragged = kAny || (V & 7);
#pragma unroll
        for (int u = 0; u < kRowVecs; ++u) {
            const int i = begin + tid + u * kRowThreads;
            if (i >= end) continue;
            const int e = 8 * i - oo;
            float2 z[4];
            widen8<kF16>(kAny && delta ? shift_entries(q[u], hi[kAny ? u : 0], delta) : q[u], z);
            if (!kBwd && bias) add_bias8(z, bias, e, V);
            shape8<kMode>(z, inv_tau, norm, a.grad_entropy != nullptr);
            store8<kMode, kF16>(dst, e, V, ragged, z, sh.mask != nullptr, allowed[u]);
        }
        __syncthreads();                                   // what follows writes over some of it
    }
    for (int k = tid; k < n_list; k += kRowThreads) store1<kMode, kF16>(dst, (s_list[k] & 0x7fff) + tb, s_val[k]);
}

// ---------------------------------------------------------------- a walk down the rows
// Where a row's vectors lie.
struct ShapeRow {
    const uint16_t* src;
    int oo;                                 // entries of the first vector that precede the row
    int delta;                              // entries by which the source is off the vectors' boundaries
    int end;                                // one past the warp's last vector
};

// kAny: rows of any alignment.  The vectors then follow the rows that are written (the source's where none are), and a source
// that is off them by `delta` entries is shifted into place from two aligned vectors.
template <int kMode, bool kF16, bool kAny>
__device__ __forceinline__ void shaping_walk(const ShapeKernelArgs& a)
{
    constexpr bool kLp = kMode == kShapeLp, kLpBwd = kMode == kShapeLpBwd, kBwd = kMode == kShapeBwd, k32 = kMode == kShape32;
    constexpr bool kTokens = kLp || kLpBwd;                // a row has a generated token
    extern __shared__ __align__(16) unsigned char smem[];
    const bool sparse = !kLp && a.sparse;
    __shared__ ShapeWalk s_w;
    __shared__ int s_scan[kShapeWarps];
    // the tokens before the coming rows: each one (less tb), the rows (bits) that it stands before, and whether H has it already
    __shared__ int s_token[kShapeRows];
    __shared__ uint32_t s_before[kShapeRows];
    __shared__ uint32_t s_fresh;
    __shared__ int s_tokens;
    __shared__ int s_y[kTokens ? kShapeRows : 1];          // the generated token (-1: out of range)
    __shared__ ShapeNorm s_norm[kLpBwd ? kShapeRows : 1];
    __shared__ float s_lp[kLpBwd ? kShapeRows : 1];
    __shared__ LpAcc s_part[kLp ? kShapeRows : 1][kLp ? kShapeWarps : 1];
    __shared__ float4 s_row[kLp ? kShapeRows : 1];         // the block's sums of a row (m, s, ez) and x of the generated token
    __shared__ float s_zy[kLp ? kShapeRows : 1];
    __shared__ long long s_count[33];
    __shared__ long long s_range[4];                       // rows the block has left: [0], [1]; padded ones: [2], [3]

    const ShapingArgs& sh = a.sh;
    const int tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, lane = tid & 31, W = nt >> 5;
    const int C = kLp ? a.cluster : 1;
    const int rank = kLp ? (int)(blockIdx.x % (unsigned)C) : 0;
    const int V = a.V, T = a.T, SV = a.segment * W;
    const int n_ent = SV * 8 + (kAny ? 16 : 0);
    const bool want_ent = kLp && a.out_entropy != nullptr;
    const int split = kLp ? 1 : a.n_slices;                // slices that are dealt to blocks (kShapeLp: to the blocks of a cluster)

    const ShapeSmem at = shape_smem(a, W, kAny);
    uint32_t* const s_bits = (uint32_t*)(smem + at.bits);        // bit k of word w: entry tb + 32 w + k is formed by itself
    uint16_t* const s_list = (uint16_t*)(smem + at.list);        // those entries, less tb
    uint8_t* const s_mark = smem + at.marks;                     // 1 + place among s_token of a listed entry that is there, or 0
    uint32_t* const s_cnt = (uint32_t*)(smem + at.counts);       // how often the answer has an entry (16 or 32 bits)
    const int buf_bytes = 16 * a.segment + (kAny ? 32 : 0), n_words = a.segment / 4 + 4;
    unsigned char* const bufs = smem + (size_t)warp * a.n_bufs * buf_bytes;
    uint32_t* const words = (uint32_t*)(smem + at.words) + warp * 2 * n_words;   // the warp's mask words of two rows
    const uint32_t bars = smem_u32(smem + at.bars) + 8u * (uint32_t)(warp * a.n_bufs);
    if (lane == 0) {
        for (int i = 0; i < a.n_bufs; ++i) mbar_init(bars + 8u * i, 1);
        fence_mbar_init();
    }
    __syncwarp();
    uint32_t phases = 0;                                   // bit i: parity of the next wait for buffer i
    bool aborted = false;

    pdl_wait_prior_grid();                                 // nothing above touches global memory
    pdl_release_next_grid();

    // ---- what the block has: a range of the list of (slice, valid row) pairs, slice by slice, or the row it is named after
    if (!a.direct) {
        const long long N = block_count_valid(a.lengths, a.B, T, s_count, nullptr);
        if (tid < 2) {
            const long long unit = blockIdx.x / (unsigned)C, units = gridDim.x / (unsigned)C;
            const long long total = (tid == 0 ? N : (long long)a.B * T - N) * split, each = total / units, rest = total % units;
            s_range[2 * tid] = unit * each + min(unit, rest);
            s_range[2 * tid + 1] = (unit + 1) * each + min(unit + 1, rest);
        }
        __syncthreads();
    }
    if (blockIdx.x == 0) report_settings(a);

    for (;;) {
        // ---- the next rows of one sequence
        int slice, t, te;
        {
            int b;
            if (a.direct) {
                const long long flat = blockIdx.x / (unsigned)C;
                b = (int)(flat / T);
                t = (int)(flat - (long long)b * T);
                te = t + 1;
                slice = rank;
                if (t >= __ldg(a.lengths + b)) break;      // padding
            } else {
                const long long k = s_range[0], N = s_count[32];
                if (k >= s_range[1]) break;
                slice = kLp ? 0 : (int)(k / N);
                const long long i = k - slice * N;
                long long before;
                find_row(a.lengths, a.B, T, false, i, b, before);
                t = (int)(i - before);
                int n = (int)min((long long)(clamp_len(__ldg(a.lengths + b), T) - t), s_range[1] - k);
                if (kLp && a.n_slices > C) n = min(n, kShapeRows);       // the sums of the rows wait for all slices
                te = t + n;
                if (kLp) slice = rank;
            }
            __syncthreads();                               // the rows before are done with the table, and all know the range
            if (tid == 0) {
                if (!a.direct) s_range[0] += te - t;
                ShapeWalk w;
                w.src = a.src + (long long)b * a.src_stride_b;
                w.logits = kBwd ? a.logits + (long long)b * a.logits_stride_b : nullptr;
                w.dst = k32 ? (void*)((float*)a.dst + (long long)b * a.dst_stride_b) : (void*)((uint16_t*)a.dst + (long long)b * a.dst_stride_b);
                w.mask = sh.mask ? sh.mask + (long long)b * sh.mask_stride_b : nullptr;
                w.bias = sh.bias ? sh.bias + (long long)b * sh.bias_stride_b : nullptr;
                w.answer = sh.tokens + (long long)b * sh.tokens_stride_b;
                w.ids = kTokens ? a.ids + (long long)b * a.ids_stride_b : nullptr;
                w.flat = (long long)b * T;
                w.ta = t;
                w.te = te;
                load_settings(sh, b, w);
                s_w = w;
            }
            __syncthreads();
        }

        for (; slice < a.n_slices; slice += kLp ? C : a.n_slices) {      // (one turn but for rows whose slices outnumber the cluster)
            const int begin = slice * SV;
            const int v0 = begin + warp * a.segment;       // the warp's first vector
            const int tb = begin * 8 - (kAny ? 8 : 0);     // entry of the table's first bit
            const float inv_tau = s_w.inv_tau;
            const bool ragged = kAny || (V & 7);
            const long long lo = max(tb, 0), span = max(min((long long)tb + n_ent, (long long)V) - lo, 0ll);
    auto in_table = [&](long long v) { return (unsigned long long)v - (unsigned long long)lo < (unsigned long long)span; };
            auto row_at = [&](int t) {
                ShapeRow r;
                r.src = s_w.src + (long long)t * a.src_stride_t;
                r.oo = r.delta = 0;
                if (kAny) {
                    const uintptr_t d = k32 ? (uintptr_t)((float*)s_w.dst + (long long)t * a.dst_stride_t)
                                            : (uintptr_t)((uint16_t*)s_w.dst + (long long)t * a.dst_stride_t);
                    r.oo = kLp ? (int)((uintptr_t)r.src >> 1) & 7 : k32 ? (int)(d >> 2) & 3 : (int)(d >> 1) & 7;
                    r.delta = ((int)((uintptr_t)r.src >> 1) - r.oo) & 7;
                }
                r.end = min(v0 + a.segment, (r.oo + V + 7) >> 3);
                return r;
            };
            // Buffer `i` gets the warp's part of a row: the 16-byte blocks of the source from that of its first vector on, as far as
            // they hold entries of the row.  (lane 0; with kAny a row may leave the last warp nothing)
            auto issue = [&](int t, int i) {
                const ShapeRow r = row_at(t);
                if (v0 >= r.end) return;
                int n = r.end - v0, skip = 0;
                if (kAny) {
                    const int e = 8 * v0 - r.oo - r.delta;             // first entry of the first block
                    if (r.delta) ++n;
                    if (e + 8 <= 0) skip = 1;
                    n = min(n, (V - e + 7) >> 3) - skip;
                }
                const uint32_t bar = bars + 8u * i;
                mbar_arrive_expect_tx(bar, 16u * (uint32_t)n);
                bulk_load(smem_u32(bufs) + (uint32_t)(i * buf_bytes + 16 * skip), r.src + (8 * (v0 + skip) - r.oo - r.delta), 16u * (uint32_t)n, bar);
            };
            // The row's mask words from that of the warp's first entry on, into the half of `words` that is not in use.
            auto issue_words = [&](int t) {
                const int w0 = (8 * v0 - (kAny ? row_at(t).oo : 0)) >> 5;
                const uint32_t* const m = s_w.mask + (long long)t * sh.mask_stride_t;
                // (16 bytes at a time for log-probs, which are bound by their instructions: 699 us where words take 785)
                if (kLp && !kAny && ((V + 31) >> 5) - w0 >= a.segment / 4 && ((uintptr_t)(m + w0) & 15) == 0) {
                    for (int i = lane; i < a.segment / 16; i += 32)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                                     ::"r"(smem_u32(words + (t & 1) * n_words + 4 * i)), "l"(m + w0 + 4 * i) : "memory");
                } else {
                    for (int i = lane; i < n_words; i += 32)
                        if (w0 + i >= 0 && w0 + i < (V + 31) >> 5)
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(words + (t & 1) * n_words + i)), "l"(m + w0 + i) : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            if (lane == 0 && !sparse)
                for (int i = 0; i < a.n_bufs && t + i < te; ++i) issue(t + i, i);
            if (sh.mask) issue_words(t);

            // ---- the history before the first row
            if (a.bits_words > 0) {
                if (kLp && slice != rank) __syncthreads(); // (a later turn: the earlier one is done with the table)
                for (int i = tid; i < a.bits_words; i += nt) s_bits[i] = 0u;
                if (a.uses_counts) {
                    const int words = a.wide_counts ? n_ent : n_ent / 2;
                    for (int i = tid; i < words / 4; i += nt) ((uint4*)s_cnt)[i] = make_uint4(0, 0, 0, 0);
                }
                if (tid == 0) s_tokens = 0;
                __syncthreads();
            }
            if (a.uses_history) {
                bool bad_id = false;
                auto mark = [&](long long v, bool of_answer) {
                    if (!in_table(v)) {
                        if (v < -1 || v >= V) bad_id = true;
                        return;
                    }
                    const int el = (int)v - tb;
                    atomicOr(s_bits + (el >> 5), 1u << (el & 31));
                    if (of_answer && a.uses_counts) {
                        if (a.wide_counts) atomicAdd(s_cnt + el, 1u);
                        else atomicAdd(s_cnt + (el >> 1), 1u << (16 * (el & 1)));
                    }
                };
                const int b = (int)(s_w.flat / T);
                const int plen = sh.prompt_lengths ? clamp_len(__ldg(sh.prompt_lengths + b), sh.P) : sh.P;
                const long long* p = sh.prompt + (long long)b * sh.prompt_stride_b;
                const int n = sh.tokens ? (int)min((long long)s_w.first + t, (long long)sh.S) : 0;
                auto scan = [&](const long long* from, int n, bool of_answer) {
                    for (int i = tid; i < n; i += 4 * nt) {
                        long long v[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) v[u] = u * nt < n - i ? __ldg(from + i + u * nt) : -1;
#pragma unroll
                        for (int u = 0; u < 4; ++u) mark(v[u], of_answer);
                    }
                };
                scan(p, plen, false);
                scan(s_w.answer, n, true);
                if (bad_id) atomicOr(a.status, kErrIdRange);
            }

            // ---- every kShapeRows rows: what the rows need beside their logits, and the tokens before them into the table
            int l0 = 0, l1 = 0;                            // the warp's part of the list
            auto begin_rows = [&](int t) {
                const int n = min(kShapeRows, te - t);
                __syncthreads();                           // the rows before are done; the bits are there
                if (a.uses_counts && tid < s_tokens) {
                    // the tokens that stood before the rows before join the counts
                    const int el = s_token[tid], more = __popc(s_before[tid]);
                    if (a.wide_counts) s_cnt[el] += more;
                    else ((uint16_t*)s_cnt)[el] += (uint16_t)more;
                }
                if (a.uses_history) __syncthreads();
                if (warp == 0 && a.uses_history) {
                    int el = -1;
                    if (sh.tokens && lane < n && t + lane > s_w.ta && (long long)s_w.first + t + lane - 1 < sh.S) {
                        const long long v = s_w.answer[s_w.first + t + lane - 1];
                        if (in_table(v)) el = (int)v - tb;
                        else if (v < -1 || v >= V) atomicOr(a.status, kErrIdRange);
                    }
                    const uint32_t same = __match_any_sync(0xffffffffu, el);
                    const bool one = el >= 0 && lane == __ffs(same) - 1;
                    const bool fresh = one && !(s_bits[el >> 5] >> (el & 31) & 1u);
                    const uint32_t all = __ballot_sync(0xffffffffu, one);
                    const int k = __popc(all & ((1u << lane) - 1u));
                    if (lane == 0) {
                        s_tokens = __popc(all);
                        s_fresh = 0u;
                    }
                    __syncwarp();
                    if (one) {
                        s_token[k] = el;
                        s_before[k] = same;
                        if (fresh) {
                            atomicOr(s_bits + (el >> 5), 1u << (el & 31));
                            atomicOr(&s_fresh, 1u << k);
                        }
                    }
                }
                if (kTokens && warp == W - 1 && lane < n) {
                    const long long y = __ldg(s_w.ids + t + lane);
                    const bool known = y >= 0 && y < V;
                    s_y[lane] = known ? (int)y : -1;
                    if (!known) atomicOr(a.status, kErrIdRange);
                    if (kLpBwd) {
                        s_norm[lane] = shape_norm(a, s_w.flat + t + lane, known, s_w.tau, inv_tau);
                        s_lp[lane] = __ldg(a.lp + s_w.flat + t + lane);
                    }
                }
                __syncthreads();
                if (!a.uses_history) return;
                // the list, from the bits: each thread its words, in order
                const int per = (a.bits_words + nt - 1) / nt, w0 = min(a.bits_words, per * tid), w1 = min(a.bits_words, w0 + per);
                int mine = 0;
                for (int w = w0; w < w1; ++w) mine += __popc(s_bits[w]);
                int upto = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += v;
                }
                if (lane == 31) s_scan[warp] = upto;
                __syncthreads();
                int before = upto - mine, n_list = 0;
                for (int w = 0; w < W; ++w) {
                    if (w < warp) before += s_scan[w];
                    n_list += s_scan[w];
                }
                for (int w = w0; w < w1; ++w)
                    for (uint32_t m = s_bits[w]; m; m &= m - 1) {
                        s_mark[before] = 0;
                        s_list[before++] = (uint16_t)(32 * w + __ffs(m) - 1);
                    }
                __syncthreads();
                auto lower = [&](int el) {                 // first place whose entry is not below el
                    int lo = 0, hi = n_list;
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if ((int)s_list[mid] < el) lo = mid + 1; else hi = mid;
                    }
                    return lo;
                };
                if (tid < s_tokens) s_mark[lower(s_token[tid])] = (uint8_t)(tid + 1);
                // (with kAny a vector begins up to seven entries early: entry_of looks whose an entry is)
                l0 = lower(8 * (v0 - begin) + (kAny ? 1 : 0));
                l1 = lower(8 * (v0 - begin + a.segment) + (kAny ? 8 : 0));
                __syncthreads();
            };

            int base = t;                                  // first row since the table was brought up to date
            int slot = 0;
            begin_rows(t);

            for (;; ++t) {
                const int r = t - base, y = kTokens ? s_y[r] : -1;
                const ShapeRow row = row_at(t);
                void* const dst = kLp ? nullptr : k32 ? (void*)((float*)s_w.dst + (long long)t * a.dst_stride_t)
                                                      : (void*)((uint16_t*)s_w.dst + (long long)t * a.dst_stride_t);
                const ShapeNorm norm = kLpBwd ? s_norm[r] : ShapeNorm{};
                const bool mine = v0 < row.end;            // (the whole warp)
                const uint32_t* const my_words = words + (t & 1) * n_words;
                const int first = 8 * v0 - row.oo;         // the warp's first entry
                if (sh.mask) {
                    asm volatile("cp.async.wait_group 0;" ::: "memory");
                    __syncwarp();
                    if (t + 1 < te) issue_words(t + 1);
                }
                const unsigned char* const buf = bufs + slot * buf_bytes;
                // the generated token, if it is the warp's and not listed
                const bool y_here = kTokens && mine && y >= max(first, 0) && y < 8 * row.end - row.oo &&
                                    !(a.uses_history && (s_bits[(y - tb) >> 5] >> ((y - tb) & 31) & 1u));
                // an entry that the lane forms by itself: those of the list and behind them (l1) the generated token; less tb, -1: none
                auto entry_of = [&](int k) {
                    if (kTokens && k == l1) return y_here ? y - tb : -1;
                    if (k >= l1) return -1;
                    const int el = s_list[k], i = (el + tb + row.oo) >> 3;
                    return i < v0 || i >= row.end ? -1 : el;
                };
                auto sign_of = [&](int el) {               // kShapeBwd: the logit, for its sign
                    return kBwd && el >= 0 ? El<kF16>::widen(__ldg(s_w.logits + (long long)t * a.logits_stride_t + el + tb)) : 0.f;
                };
                // such an entry
                auto form = [&](int k, int el, float sign) {
                    const int v = el + tb;
                    // a token of the coming rows is listed ahead of its time
                    const uint32_t j = k < l1 ? s_mark[k] : 0u;
                    const uint32_t so_far = j ? s_before[j - 1] & ((2u << r) - 1u) : 0u;
                    const bool listed = k < l1 && (so_far || !(j && (s_fresh >> (j - 1) & 1u)));
                    const float raw = El<kF16>::widen(sparse ? row.src[v] : ((const uint16_t*)buf)[v - (first - row.delta)]);
                    const bool ok = !sh.mask || (my_words[(v >> 5) - (first >> 5)] >> (v & 31) & 1u);
                    uint32_t c = 0;
                    if (a.uses_counts && listed) c = (a.wide_counts ? s_cnt[el] : ((const uint16_t*)s_cnt)[el]) + __popc(so_far);
                    return shape1<kMode>(raw, listed ? ((kBwd ? sign : raw) < 0.f ? s_w.rep : s_w.inv_rep) : 1.f, c, s_w.freq, s_w.pres,
                                         sh.bias ? s_w.bias + v : nullptr, ok, kLp ? s_w.inv_tau : inv_tau, norm, a.grad_entropy != nullptr,
                                         kLpBwd && v == y, kLpBwd ? s_lp[r] : 0.f);
                };
                int el = mine && !kLp ? entry_of(l0 + lane) : -1;
                float sign = sign_of(el);                  // (in flight during the row)
                if (kLp && y_here) {                       // (left out of the sum as the listed are)
                    __syncwarp();
                    if (lane == 0) atomicOr(s_bits + ((y - tb) >> 5), 1u << ((y - tb) & 31));
                    __syncwarp();
                }

                LaneSums acc = lane_sums();
                const float k2 = kLog2e * inv_tau;
                if (mine && !sparse) {
                    mbar_wait_here(bars + 8u * slot, (phases >> slot) & 1u, a.status, aborted, a.wait_limit_ns);
                    phases ^= 1u << slot;
                    const uint4* const vecs = (const uint4*)buf;
                    const int n = row.end - v0;
                    auto vec = [&](int i) {                // i: of the warp's vectors
                        return kAny && row.delta ? shift_entries(vecs[i], vecs[i + 1], row.delta) : vecs[i];
                    };
                    auto marks = [&](int i) -> uint32_t {  // its mask
                        if (!kAny) return ((const uint8_t*)my_words)[i];
                        const int x = (first & 31) + 8 * i;
                        return __funnelshift_r(my_words[x >> 5], my_words[(x >> 5) + 1], x & 31);
                    };
                    if (kLp) {
                        // two vectors at a time, what is not summed at -inf
                        if (!kAny && !sh.bias && n == a.segment && first + 8 * n <= V) {
                            // (what aligned rows need and nothing else: the loop is bound by its instructions)
                            uint32_t pv = smem_u32(buf) + 16u * lane, pb = smem_u32(s_bits) + (uint32_t)(v0 - begin + lane), pm = smem_u32(my_words) + lane;
                            auto stream = [&](auto masked, auto entropy) {
#pragma unroll 1
                                for (const uint32_t pe = pv + 16u * (uint32_t)a.segment; pv < pe; pv += 1024u, pb += 64u, pm += 64u) {
                                    float2 z[2][4];
#pragma unroll
                                    for (int u = 0; u < 2; ++u) {
                                        uint4 w;
                                        uint32_t drop, allow = ~0u;
                                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(pv + 512u * u) : "memory");
                                        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(drop) : "r"(pb + 32u * u) : "memory");
                                        if (decltype(masked)::value) asm volatile("ld.shared.u8 %0, [%1];" : "=r"(allow) : "r"(pm + 32u * u) : "memory");
                                        widen8<kF16>(keep_entries(w, allow & ~drop, El<kF16>::kNegInf2), z[u]);
                                    }
                                    lane_add16(acc, z, k2, decltype(entropy)::value);
                                }
                            };
                            if (sh.mask) {
                                if (want_ent) stream(std::true_type{}, std::true_type{}); else stream(std::true_type{}, std::false_type{});
                            } else {
                                if (want_ent) stream(std::false_type{}, std::true_type{}); else stream(std::false_type{}, std::false_type{});
                            }
                        } else {
                        auto turn = [&](int i, auto kind) {
                            constexpr bool whole = decltype(kind)::value;
                            float2 z[2][4];
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                int x = i + 32 * u;
                                const bool in = whole || x < n;
                                if (!in) x = 0;
                                uint32_t keep;
                                if (!kAny) {
                                    keep = ~(uint32_t)((const uint8_t*)s_bits)[(v0 - begin) + x];
                                } else {
                                    const int e = first + 8 * x - tb;
                                    keep = ~__funnelshift_r(s_bits[e >> 5], s_bits[(e >> 5) + 1], e & 31);
                                }
                                if (sh.mask) keep &= marks(x);
                                if (!whole) {
                                    const int e = first + 8 * x;
                                    if (e < 0) keep &= ~0u << -e;
                                    if (e + 8 > V) keep &= (1u << max(0, V - e)) - 1u;
                                    if (!in) keep = 0u;
                                }
                                uint4 w = vec(x);
                                if ((keep & 0xffu) != 0xffu) w = keep_entries(w, keep, El<kF16>::kNegInf2);
                                widen8<kF16>(w, z[u]);
                                if (sh.bias) {
                                    float b[8];
                                    load_bias(s_w.bias, first + 8 * x, V, b);
#pragma unroll
                                    for (int j = 0; j < 4; ++j)        // (what is left out stays -inf, whatever its bias)
                                        z[u][j] = __fadd2_rn(z[u][j], make_float2(keep >> (2 * j) & 1u ? b[2 * j] : 0.f, keep >> (2 * j + 1) & 1u ? b[2 * j + 1] : 0.f));
                                }
                            }
                            lane_add16(acc, z, k2, want_ent);
                        };
                        if (n == a.segment && first >= 0 && first + 8 * n <= V) {
                            for (int i = lane; i < a.segment; i += 64) turn(i, std::true_type{});
                        } else {
                            for (int i = lane; i - lane < n; i += 64) turn(i, std::false_type{});
                        }
                        }
                    } else {
#pragma unroll 2
                        for (int i = lane; i < n; i += 32) {
                            float2 z[4];
                            widen8<kF16>(vec(i), z);
                            if (!kBwd && sh.bias) add_bias8(z, s_w.bias, first + 8 * i, V);
                            shape8<kMode>(z, inv_tau, norm, a.grad_entropy != nullptr);
                            store8<kMode, kF16>(dst, first + 8 * i, V, ragged, z, sh.mask != nullptr, sh.mask ? marks(i) : ~0u);
                        }
                    }
                }

                // ---- the entries that are formed by themselves
                if (mine) {
                    __syncwarp();                          // (what follows writes over what the stream of vectors wrote)
                    const int last = l1 + (y_here ? 1 : 0);
                    if (kLp) el = entry_of(l0 + lane);
                    for (int k = l0 + lane; k - lane < last;) {
                        if (el >= 0) {
                            const float x = form(k, el, sign);
                            if (!kLp) store1<kMode, kF16>(dst, el + tb, x);
                            else if (el + tb == y) s_zy[r] = x * s_w.inv_tau;
                            else lane_add1(acc, x, k2, want_ent);
                        }
                        k += 32;
                        if (k - lane >= last) break;
                        el = entry_of(k);                  // (a warp with more than 32 such entries)
                        sign = sign_of(el);
                    }
                    if (kLp && y_here && lane == 0) atomicAnd(s_bits + ((y - tb) >> 5), ~(1u << ((y - tb) & 31)));
                    __syncwarp();                          // every lane is done with the buffer
                }
                if (!sparse) {
                    if (lane == 0 && t + a.n_bufs < te) issue(t + a.n_bufs, slot);
                    slot = slot + 1 == a.n_bufs ? 0 : slot + 1;
                }

                if (kLp) {
                    const LpAcc mine = lane_done(acc, k2, s_w.inv_tau);
                    const float M = warp_max(mine.m);
                    const float up = M - mine.m, sc = ex2(-up * kLog2e);
                    float s = mine.s * sc, ez = sc * (mine.ez - up * mine.s);
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) {
                        s += __shfl_xor_sync(0xffffffffu, s, o);
                        if (want_ent) ez += __shfl_xor_sync(0xffffffffu, ez, o);
                    }
                    if (lane == 0) {
                        LpAcc& part = s_part[r][warp];
                        part = slice < C ? LpAcc{M, s, ez} : lp_merge(part, LpAcc{M, s, ez});
                    }
                    if ((t + 1 >= te || r + 1 == kShapeRows) && slice + C >= a.n_slices) {
                        // the block's sums of the rows, then the cluster's
                        __syncthreads();
                        for (int i = warp; i <= r; i += W) {
                            LpAcc p = lane < W ? s_part[i][lane] : LpAcc{kFloorM, 0.f, 0.f};
#pragma unroll
                            for (int o = 16; o > 0; o >>= 1)
                                p = lp_merge(p, LpAcc{__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                                                      __shfl_xor_sync(0xffffffffu, p.ez, o)});
                            if (lane == 0) s_row[i] = make_float4(p.m, p.s, p.ez, s_zy[i]);
                        }
                        __syncthreads();
                        if (C > 1) {
                            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
                            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
                        }
                        if (rank == 0 && tid <= r) {
                            const int yy = s_y[tid];
                            // the block that has seen the generated token
                            const int off = kAny ? (int)((uintptr_t)(s_w.src + (long long)(base + tid) * a.src_stride_t) >> 1) & 7 : 0;
                            lp_finish(a, s_row + tid, yy, yy >= 0 ? ((off + yy) >> 3) / SV % C : 0, C, s_w.flat + base + tid);
                        }
                        if (C > 1) {                       // the others' rows have been read
                            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
                            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
                        }
                    }
                }
                if (t + 1 >= te) break;
                if (r + 1 == kShapeRows) {
                    base = t + 1;
                    begin_rows(t + 1);
                }
            }
            t = s_w.ta;
        }
        if (a.direct) break;
    }

    // ---- padding
    if (!kLp) {
        const long long pads = (long long)a.B * T - s_count[32];
        for (long long k = s_range[2]; k < s_range[3];) {
            const int slice = (int)(k / pads);
            int b;
            long long before;
            find_row(a.lengths, a.B, T, true, k - slice * pads, b, before);
            const int t = clamp_len(__ldg(a.lengths + b), T) + (int)(k - slice * pads - before);
            const int n = (int)min((long long)(T - t), s_range[3] - k);
            const long long off = (long long)b * a.dst_stride_b;
            clear_rows<k32, kAny>(k32 ? (void*)((float*)a.dst + off) : (void*)((uint16_t*)a.dst + off), a.dst_stride_t, t, t + n, slice * SV, SV, V);
            k += n;
        }
    } else {
        const long long total = (long long)a.B * T;
        for (long long i = (long long)blockIdx.x * nt + tid; i < total; i += (long long)gridDim.x * nt) {
            const int b = (int)(i / T), t = (int)(i - (long long)b * T);
            if (t < __ldg(a.lengths + b)) continue;
            a.out_lp[i] = 0.f;
            *((float2*)a.out_lse + i) = make_float2(0.f, 0.f);
            if (a.out_entropy) a.out_entropy[i] = 0.f;
        }
    }
}

template <int kMode, bool kF16, bool kAny>
__global__ void __launch_bounds__(kShapeWarps * 32, 1) shaping_kernel(const __grid_constant__ ShapeKernelArgs a)
{
    shaping_walk<kMode, kF16, kAny>(a);
}
template <bool kF16, bool kAny>
__global__ void __launch_bounds__(kShapeLpWarps * 32, 1) shaping_lp_kernel(const __grid_constant__ ShapeKernelArgs a)
{
    shaping_walk<kShapeLp, kF16, kAny>(a);
}

}  // namespace rlhf
