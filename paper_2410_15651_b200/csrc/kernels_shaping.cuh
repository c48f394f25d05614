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
// and walks down its rows; each of its warps has a segment of the slice (at most 256 vectors of eight entries), a ring of buffers
// that bulk copies fill a few rows ahead, and nothing to wait for but its own buffers.  In shared memory the block has a bit
// per entry that says "in H, or will be within the coming 32 rows", the ascending list of those entries and, where penalties count,
// c_v of every entry; they are built where a block begins a sequence and brought up to date every 32 rows.  A warp streams its
// segment of a row as if no entry were in H, and then forms those that are (one or two per lane) by themselves, from the
// same buffer: it writes them over what the stream wrote, or, where a sum is wanted, the stream has left them out.  The generated token is
// formed apart in the same way.  Bits and counts come from atomics on whole numbers, so no result depends on their order.
#pragma once
#include "async.cuh"
#include "common.cuh"

namespace rlhf {

constexpr unsigned kErrValueRange = 128u;

constexpr int kShapeWarps = 16;             // warps of a block, at most
constexpr int kShapeSegment = 256;          // vectors of eight entries of a warp, at most
constexpr int kShapeRows = 32;              // rows between two updates of the table
constexpr int kShapeMaxCluster = 8;
constexpr int kShapeDirectRows = 16;        // shorter sequences have a block for each row
constexpr int kShapeMaxBufs = 4;

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
    int direct;                             // a block (cluster) per row, padded ones too, instead of a range of the valid rows
    int bits_words;                         // words of the bit table in shared memory
    int list_cap;                           // entries of the list
    int uses_history, uses_counts;
    int wide_counts;                        // counts of 32 instead of 16 bits
    int sparse;                             // in place and nothing but penalties: only entries of H are touched
};

// Shared memory, in this order: the warps' buffers, their barriers, the bits, the list, the list's marks, the counts.
struct ShapeSmem {
    size_t bufs, bars, bits, list, marks, counts, total;
};
__host__ __device__ inline ShapeSmem shape_smem(const ShapeKernelArgs& a, int warps, bool any)
{
    const size_t buf = 16 * (size_t)a.segment + (any ? 32 : 0), entries = 8 * (size_t)a.segment * warps + (any ? 16 : 0);
    ShapeSmem s;
    s.bufs = 0;
    s.bars = s.bufs + (a.sparse ? 0 : buf * warps * a.n_bufs);
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
    float rep, inv_rep, freq, pres, inv_tau;
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

// Adds eight terms to a partial sum.
__device__ __forceinline__ void lp_add8(LpAcc& acc, const float2 (&z)[4], float scale, bool want_ent)
{
    float2 d[4], e[4];
    float vs;
    auto sums = [&]() {
        const float2 nm = splat2(-acc.m), sc = splat2(scale), l2 = splat2(kLog2e);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            d[j] = __ffma2_rn(z[j], sc, nm);
            const float2 y = __fmul2_rn(d[j], l2);
            e[j] = make_float2(ex2(y.x), ex2(y.y));
        }
        const float2 a = __fadd2_rn(__fadd2_rn(e[0], e[1]), __fadd2_rn(e[2], e[3]));
        vs = a.x + a.y;
    };
    if (acc.m == kFloorM) {                                // the first of a row: its own maximum (where it has one)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc.m = fmaxf(acc.m, fmaxf(z[j].x * scale, z[j].y * scale));
    }
    sums();
    if (!(vs <= 1.8446744e19f)) {
        // a term more than 64 binades above the reference
        float m = kFloorM;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, fmaxf(z[j].x * scale, z[j].y * scale));
        const float up = m - acc.m, c = ex2(-up * kLog2e);
        acc.ez = c * (acc.ez - up * acc.s);
        acc.s *= c;
        acc.m = m;
        sums();
    }
    acc.s += vs;
    if (want_ent) {
        float2 v = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v = __ffma2_rn(e[j], make_float2(fmaxf(d[j].x, kLpClamp), fmaxf(d[j].y, kLpClamp)), v);
        acc.ez += v.x + v.y;
    }
}

// One term, for the entries that are formed by themselves.
__device__ __forceinline__ void lp_add1(LpAcc& acc, float x, bool want_ent)
{
    if (x - acc.m > 44.f) {
        const float up = x - acc.m, c = ex2(-up * kLog2e);
        acc.ez = c * (acc.ez - up * acc.s);
        acc.s *= c;
        acc.m = x;
    }
    const float d = x - acc.m, e = ex2(d * kLog2e);
    acc.s += e;
    if (want_ent) acc.ez = fmaf(e, fmaxf(d, kLpClamp), acc.ez);
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
    if (a.out_entropy) a.out_entropy[flat] = total > 0.f ? lo - (p.ez + ey * fmaxf(dy, kLpClamp)) / total : 0.f;
}

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
__global__ void __launch_bounds__(kShapeWarps * 32, 1) shaping_kernel(const __grid_constant__ ShapeKernelArgs a)
{
    constexpr bool kLp = kMode == kShapeLp, kLpBwd = kMode == kShapeLpBwd, kBwd = kMode == kShapeBwd, k32 = kMode == kShape32;
    constexpr bool kTokens = kLp || kLpBwd;                // a row has a generated token
    constexpr uint32_t kOut2 = kBwd || kLpBwd ? 0u : El<kF16>::kNegInf2;       // what a masked entry gives
    constexpr int kTurns = kShapeSegment / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ ShapeWalk s_w;
    __shared__ int s_scan[kShapeWarps];
    // the tokens before the coming rows: each one (less tb), the rows (bits) that it stands before, and whether H has it already
    __shared__ int s_token[kShapeRows];
    __shared__ uint32_t s_before[kShapeRows];
    __shared__ uint32_t s_fresh;
    __shared__ int s_tokens;
    __shared__ int s_y[kTokens ? kShapeRows : 1];          // the generated token (-1: out of range)
    __shared__ float4 s_norm[kLpBwd ? kShapeRows : 1];     // less the normaliser's parts, less the gradients over tau
    __shared__ float2 s_more[kLpBwd ? kShapeRows : 1];     // entropy, log-prob
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
    uint32_t* const s_bits = (uint32_t*)(smem + at.bits);        // bit k of word w: entry tb + 32 w + k is listed
    uint16_t* const s_list = (uint16_t*)(smem + at.list);        // listed entries, less tb
    uint8_t* const s_mark = smem + at.marks;                     // 1 + place among s_token of a listed entry that is there, or 0
    uint32_t* const s_cnt = (uint32_t*)(smem + at.counts);       // how often the answer has an entry (16 or 32 bits)
    const int buf_bytes = 16 * a.segment + (kAny ? 32 : 0);
    unsigned char* const bufs = smem + (size_t)warp * a.n_bufs * buf_bytes;
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

    // ---- what is wrong with the sequences' numbers, said once
    if (blockIdx.x == 0) {
        unsigned wrong = 0;
        for (int b = tid; b < a.B; b += nt) {
            const int n = __ldg(a.lengths + b);
            if (n < 0 || n > T) wrong |= kErrLengthRange;
            const int f = sh.start ? __ldg(sh.start + b) : 0;
            if (f < 0 || (sh.tokens && n > 0 && (long long)f + min(n, T) - 1 > sh.S)) wrong |= kErrLengthRange;
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

    for (;;) {
        // ---- the next rows of one sequence
        int slice, t, te;
        {
            int b;
            if (a.direct) {
                const long long unit = blockIdx.x / (unsigned)C, flat = unit / split;
                b = (int)(flat / T);
                t = (int)(flat - (long long)b * T);
                te = t + 1;
                slice = kLp ? rank : (int)(unit - flat * split);
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
                w.first = sh.start ? max(0, __ldg(sh.start + b)) : 0;
                w.ta = t;
                w.te = te;
                // settings; one that is out of range is neutral
                float rep = sh.repetition ? __ldg(sh.repetition + b) : 1.f, tau = sh.temperature ? __ldg(sh.temperature + b) : 1.f;
                if (!(rep >= 1e-3f && rep <= 1e18f)) rep = 1.f;
                if (!(tau >= 1e-3f && tau <= 1e18f)) tau = 1.f;
                w.rep = rep;
                w.inv_rep = 1.f / rep;
                w.inv_tau = 1.f / tau;
                w.freq = sh.frequency ? __ldg(sh.frequency + b) : 0.f;
                w.pres = sh.presence ? __ldg(sh.presence + b) : 0.f;
                if (!(fabsf(w.freq) <= 1e18f)) w.freq = 0.f;
                if (!(fabsf(w.pres) <= 1e18f)) w.pres = 0.f;
                s_w = w;
            }
            __syncthreads();
            if (a.direct && t >= __ldg(a.lengths + b)) {   // padding
                if (!kLp) clear_rows<k32, kAny>(s_w.dst, a.dst_stride_t, t, te, slice * SV, SV, V);
                break;
            }
        }

        for (; slice < a.n_slices; slice += kLp ? C : a.n_slices) {      // (one turn but for rows whose slices outnumber the cluster)
            const int begin = slice * SV;
            const int v0 = begin + warp * a.segment;       // the warp's first vector
            const int tb = begin * 8 - (kAny ? 8 : 0);     // entry of the table's first bit
            const float inv_tau = s_w.inv_tau;
            auto in_table = [&](long long v) { return v >= max(tb, 0) && v < (long long)tb + n_ent && v < V; };
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
            // they hold entries of the row.  (lane 0)
            auto issue = [&](const ShapeRow& r, int i) {
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
            if (lane == 0 && !a.sparse)
                for (int i = 0; i < a.n_bufs && t + i < te; ++i) {
                    const ShapeRow r = row_at(t + i);
                    if (v0 < r.end) issue(r, i);           // (with kAny a row may leave the last warp nothing)
                }
            int next = min(te, t + a.n_bufs);              // the next row to ask for

            // ---- the history before the first row
            if (a.uses_history) {
                if (kLp && slice != rank) __syncthreads(); // (a later turn: the earlier one is done with the table)
                for (int i = tid; i < a.bits_words; i += nt) s_bits[i] = 0u;
                if (a.uses_counts) {
                    const int words = a.wide_counts ? n_ent : n_ent / 2;
                    for (int i = tid; i < words / 4; i += nt) ((uint4*)s_cnt)[i] = make_uint4(0, 0, 0, 0);
                }
                if (tid == 0) s_tokens = 0;
                __syncthreads();
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
                for (int i = tid; i < plen; i += nt) mark(__ldg(p + i), false);
                for (int i = tid; i < n; i += nt) mark(__ldg(s_w.answer + i), true);
                if (bad_id) atomicOr(a.status, kErrIdRange);
            }

            // ---- every kShapeRows rows: what the rows need beside their logits, and the tokens before them into the table
            int l0 = 0, l1 = 0;                            // the warp's part of the list
            auto begin_rows = [&](int t) {
                const int n = min(kShapeRows, te - t);
                __syncthreads();                           // the rows before are done; the bits are there
                if (a.uses_history && a.uses_counts && tid < s_tokens) {
                    // the tokens that stood before the rows before join the counts
                    const int el = s_token[tid], more = __popc(s_before[tid]);
                    if (a.wide_counts) s_cnt[el] += more;
                    else ((uint16_t*)s_cnt)[el] += (uint16_t)more;
                }
                if (a.uses_history) __syncthreads();
                if (warp == 0 && a.uses_history) {
                    int el = -1;
                    if (sh.tokens && lane < n && t + lane > s_w.ta && (long long)s_w.first + t + lane - 1 < sh.S) {
                        const long long v = __ldg(s_w.answer + s_w.first + t + lane - 1);
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
                        const long long flat = s_w.flat + t + lane;
                        const float2 l = __ldg((const float2*)a.lse + flat);
                        const float h = a.grad_entropy ? __ldg(a.grad_entropy + flat) : 0.f;
                        // (a row that is all -inf has p = 0)
                        s_norm[lane] = make_float4(-l.x, l.y == -INFINITY ? 0.f : -l.y, known ? -__ldg(a.grad_lp + flat) * inv_tau : 0.f, -h * inv_tau);
                        s_more[lane] = make_float2(a.grad_entropy ? __ldg(a.entropy + flat) : 0.f, __ldg(a.lp + flat));
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
                // (with kAny a vector begins up to seven entries early: form() looks whose an entry is)
                l0 = lower(8 * (v0 - begin) + (kAny ? 1 : 0));
                l1 = lower(8 * (v0 - begin + a.segment) + (kAny ? 8 : 0));
                __syncthreads();
            };

            LpAcc acc{kFloorM, 0.f, 0.f};
            int base = t;                                  // first row since the table was brought up to date
            int slot = 0;
            uint32_t marks[kTurns] = {};                   // mask bytes of the lane's vectors, asked for a row ahead
            auto ask_marks = [&](const ShapeRow& r, int t) {
                const uint32_t* m = s_w.mask + (long long)t * sh.mask_stride_t;
#pragma unroll
                for (int u = 0; u < kTurns; ++u) {
                    const int i = v0 + lane + 32 * u;
                    if (i < r.end) {
                        if (!kAny) {
                            marks[u] = __ldg((const uint8_t*)m + i);
                        } else {
                            const int e = 8 * i - r.oo, w = e >> 5;
                            const uint32_t lo = w >= 0 ? __ldg(m + w) : 0u, hi = (e & 31) > 24 && w + 1 < (V + 31) >> 5 ? __ldg(m + w + 1) : 0u;
                            marks[u] = __funnelshift_r(lo, hi, e & 31);
                        }
                    }
                }
            };
            ShapeRow row = row_at(t);
            if (sh.mask && !a.sparse) ask_marks(row, t);
            begin_rows(t);

            for (;; ++t) {
                const int r = t - base, y = kTokens ? s_y[r] : -1;
                char* const dst = kLp ? nullptr : k32 ? (char*)((float*)s_w.dst + (long long)t * a.dst_stride_t)
                                                      : (char*)((uint16_t*)s_w.dst + (long long)t * a.dst_stride_t);
                const int yvec = kTokens && y >= 0 ? (y + row.oo) >> 3 : -1;
                float4 norm{0.f, 0.f, 0.f, 0.f};
                float ent = 0.f;
                if (kLpBwd) {
                    norm = s_norm[r];
                    ent = s_more[r].x;
                }
                const bool mine = v0 < row.end;            // (the whole warp)
                // the lane's first entry that is formed by itself: those of the list, then the generated token
                auto entry_of = [&](int k) {               // less tb; -1: none
                    int el = -1;
                    if (k < l1) el = s_list[k];
                    else if (kTokens && k == l1 && in_table(y)) {
                        el = y - tb;
                        if (a.uses_history && (s_bits[el >> 5] >> (el & 31) & 1u)) el = -1;
                    }
                    if (el >= 0) {
                        const int i = (el + tb + row.oo) >> 3;
                        if (i < v0 || i >= row.end) el = -1;
                    }
                    return el;
                };
                int el = -1;
                uint32_t word = ~0u;
                float sign = 0.f;
                auto ask = [&](int k) {
                    el = entry_of(k);
                    if (el < 0) return;
                    if (sh.mask) word = __ldg(s_w.mask + (long long)t * sh.mask_stride_t + ((el + tb) >> 5));
                    if (kBwd) sign = El<kF16>::widen(__ldg(s_w.logits + (long long)t * a.logits_stride_t + el + tb));
                };
                if (mine) ask(l0 + lane);

                const unsigned char* buf = bufs + slot * buf_bytes;
                if (mine && !a.sparse) {
                    mbar_wait(bars + 8u * slot, (phases >> slot) & 1u, a.status, aborted, a.wait_limit_ns);
                    phases ^= 1u << slot;
                    const uint4* vecs = (const uint4*)buf - v0;
#pragma unroll
                    for (int u = 0; u < kTurns; ++u) {
                        const int i = v0 + lane + 32 * u;
                        if (32 * u >= a.segment) break;
                        if (i >= row.end) continue;
                        const int e = 8 * i - row.oo;
                        uint4 w = vecs[i];
                        if (kAny && row.delta) w = shift_entries(w, vecs[i + 1], row.delta);
                        uint32_t allowed = sh.mask ? marks[u] : ~0u;
                        if (kLp) {
                            uint32_t skip = 0;
                            if (a.uses_history) {
                                if (!kAny) {
                                    skip = ((const uint8_t*)s_bits)[i - begin];
                                } else {
                                    const int b0 = e - tb;
                                    skip = __funnelshift_r(s_bits[b0 >> 5], s_bits[(b0 >> 5) + 1], b0 & 31);
                                }
                            }
                            if (i == yvec) skip |= 1u << ((y + row.oo) & 7);
                            allowed &= ~skip;
                            if (e < 0) allowed &= ~0u << -e;
                            if (e + 8 > V) allowed &= (1u << (V - e)) - 1u;
                            if ((allowed & 0xffu) != 0xffu) w = keep_entries(w, allowed, El<kF16>::kNegInf2);
                        } else if (k32 && sh.mask) {
                            w = keep_entries(w, allowed, kOut2);
                        }
                        float2 z[4] = {El<kF16>::unpack2(w.x), El<kF16>::unpack2(w.y), El<kF16>::unpack2(w.z), El<kF16>::unpack2(w.w)};
                        if (!kBwd && sh.bias) {
                            const float* bias = s_w.bias + e;
                            float b8[8];
                            if (e >= 0 && e + 8 <= V && ((uintptr_t)bias & 15) == 0) {
                                const float4 f = __ldg((const float4*)bias), g = __ldg((const float4*)bias + 1);
                                b8[0] = f.x; b8[1] = f.y; b8[2] = f.z; b8[3] = f.w; b8[4] = g.x; b8[5] = g.y; b8[6] = g.z; b8[7] = g.w;
                            } else {
#pragma unroll
                                for (int j = 0; j < 8; ++j) b8[j] = e + j >= 0 && e + j < V ? __ldg(bias + j) : 0.f;
                            }
                            if (kLp || k32) {              // (what is left out stays -inf, whatever its bias)
#pragma unroll
                                for (int j = 0; j < 8; ++j) b8[j] = allowed >> j & 1u ? b8[j] : 0.f;
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) z[j] = __fadd2_rn(z[j], make_float2(b8[2 * j], b8[2 * j + 1]));
                        }
                        if (kLp) {
                            lp_add8(acc, z, inv_tau, want_ent);
                            continue;
                        }
                        if (kLpBwd) {
                            // dx_v = -p_v (g + h (log p_v + H))
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float2 lq = __fadd2_rn(__ffma2_rn(z[j], splat2(inv_tau), splat2(norm.x)), splat2(norm.y));
                                const float2 x = __fmul2_rn(lq, splat2(kLog2e));
                                const float2 p = make_float2(ex2(x.x), ex2(x.y));
                                float2 f = splat2(norm.z);
                                if (a.grad_entropy) {
                                    const float2 k = __fadd2_rn(make_float2(fmaxf(lq.x, kLpClamp), fmaxf(lq.y, kLpClamp)), splat2(ent));
                                    f = __ffma2_rn(k, splat2(norm.w), f);
                                }
                                z[j] = __fmul2_rn(p, f);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j) z[j] = __fmul2_rn(z[j], splat2(inv_tau));
                        }
                        const bool whole = e >= 0 && e + 8 <= V;
                        if (k32) {
                            float* o = (float*)dst + e;
                            if (whole) {
                                __stcs((float4*)o, make_float4(z[0].x, z[0].y, z[1].x, z[1].y));
                                __stcs((float4*)o + 1, make_float4(z[2].x, z[2].y, z[3].x, z[3].y));
                            } else {
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    if (e + j >= 0 && e + j < V) o[j] = j & 1 ? z[j >> 1].y : z[j >> 1].x;
                            }
                            continue;
                        }
                        uint4 out = make_uint4(El<kF16>::pack2(z[0].x, z[0].y), El<kF16>::pack2(z[1].x, z[1].y),
                                               El<kF16>::pack2(z[2].x, z[2].y), El<kF16>::pack2(z[3].x, z[3].y));
                        if (sh.mask) out = keep_entries(out, allowed, kOut2);
                        uint16_t* o = (uint16_t*)dst + e;
                        if (whole) {
                            __stcs((uint4*)o, out);
                        } else {
                            const uint32_t ww[4] = {out.x, out.y, out.z, out.w};
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (e + j >= 0 && e + j < V) o[j] = (uint16_t)(ww[j >> 1] >> (16 * (j & 1)));
                        }
                    }
                }
                const ShapeRow now = row;
                if (t + 1 < te) {
                    row = row_at(t + 1);
                    if (sh.mask && !a.sparse) ask_marks(row, t + 1);
                }

                // ---- the entries that are formed by themselves
                if (mine) {
                    __syncwarp();                          // (what follows writes over what the stream of vectors wrote)
                    for (int k = l0 + lane;;) {
                        if (el >= 0) {
                            const int v = el + tb;
                            // a token of the coming rows is listed ahead of its time
                            const uint32_t j = k < l1 && s_tokens ? s_mark[k] : 0u;
                            const uint32_t so_far = j ? s_before[j - 1] & ((2u << r) - 1u) : 0u;
                            const bool listed = k < l1 && (so_far || !(j && (s_fresh >> (j - 1) & 1u)));
                            const float raw = a.sparse ? El<kF16>::widen(now.src[v])
                                                       : El<kF16>::widen(((const uint16_t*)buf)[v - (8 * v0 - now.oo - now.delta)]);
                            const bool ok = word >> (v & 31) & 1u;
                            const float by = listed ? ((kBwd ? sign : raw) < 0.f ? s_w.rep : s_w.inv_rep) : 1.f;
                            if (kBwd) {
                                ((uint16_t*)dst)[v] = (uint16_t)El<kF16>::pack2(ok ? raw * by * inv_tau : 0.f, 0.f);
                            } else {
                                float x = raw * by;
                                if (a.uses_counts && listed) {
                                    const uint32_t c = (a.wide_counts ? s_cnt[el] : ((const uint16_t*)s_cnt)[el]) + __popc(so_far);
                                    if (c > 0) x = fmaf(-s_w.freq, (float)c, x) - s_w.pres;
                                }
                                if (sh.bias) x += __ldg(s_w.bias + v);
                                x = ok ? x * inv_tau : -INFINITY;
                                if (kMode == kShape16) {
                                    ((uint16_t*)dst)[v] = (uint16_t)El<kF16>::pack2(x, 0.f);
                                } else if (k32) {
                                    ((float*)dst)[v] = x;
                                } else if (kLp) {
                                    if (v == y) s_zy[r] = x;
                                    else lp_add1(acc, x, want_ent);
                                } else {
                                    const float lq = (x + norm.x) + norm.y, p = ex2(lq * kLog2e);
                                    float d = norm.z * (v == y ? expm1f(s_more[r].y) : p);         // 1 - p without cancellation
                                    if (a.grad_entropy) d = fmaf(norm.w * p, fmaxf(lq, kLpClamp) + ent, d);
                                    d = x == -INFINITY ? 0.f : d * by;
                                    ((uint16_t*)dst)[v] = (uint16_t)El<kF16>::pack2(d, 0.f);
                                }
                            }
                        }
                        k += 32;
                        if (k >= l1 + (kTokens ? 1 : 0)) break;
                        // (rows whose warp has more than 32 such entries)
                        {
                            const ShapeRow keep = row;
                            row = now;
                            ask(k);
                            row = keep;
                        }
                    }
                    __syncwarp();                          // every lane is done with the buffer
                }
                if (!a.sparse) {
                    if (next < te) {
                        if (lane == 0) {
                            const ShapeRow n = row_at(next);
                            if (v0 < n.end) issue(n, slot);
                        }
                        ++next;
                    }
                    slot = slot + 1 == a.n_bufs ? 0 : slot + 1;
                }

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
                        LpAcc& part = s_part[r][warp];
                        part = slice < C ? LpAcc{M, s, ez} : lp_merge(part, LpAcc{M, s, ez});
                    }
                    acc = LpAcc{kFloorM, 0.f, 0.f};
                    if ((t + 1 >= te || r + 1 == kShapeRows) && slice + C >= a.n_slices) {
                        // the block's sums of the rows, then the cluster's
                        __syncthreads();
                        for (int i = warp; i <= r; i += W) {
                            LpAcc p = lane < W ? s_part[i][lane] : LpAcc{kFloorM, 0.f, 0.f};
#pragma unroll
                            for (int o = kShapeWarps / 2; o > 0; o >>= 1)
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
    if (!kLp && !a.direct) {
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
    }
    if (kLp) {
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

}  // namespace rlhf
