// Loss forward/backward with the row's exponentials kept on chip between the two passes, for 16-byte
// aligned rows of 16 KB and more; rows that do not fit one block twice are shared by a thread-block
// cluster of up to 4 blocks.
// (kernels_cring.cuh holds the variant that passes the row through a ring of chunks, which takes some row
// lengths with fewer blocks; the helpers below serve both.)
//
// A row's gradient needs every softmax term twice: once in the partition sum and once, scaled by the
// token's g / sum, as the gradient entry itself.  Recomputing the exponential in the second pass costs two
// ex2 per logit, which makes the special-function unit (16 results per clock per SM) the limiter
// whenever the SM clock drops under the power cap.  Here every consumer
// thread keeps the exponentials of its share of the row after the first pass -- those of its first
// kRegVecs vectors in registers, those of the following ones in tensor memory (the 256 KB per SM that
// otherwise hold tensor-core accumulators; each warp stores and loads its own 32 lanes x 128 columns with
// tcgen05.st / tcgen05.ld) -- so the second pass is one packed multiply and one conversion per pair of
// logits: one ex2 per logit in total, and no second read of the row from shared memory.
//
// Rows up to about 105 KB are held by one block, in two row buffers (three where they fit, which keeps more
// loads in flight): while row i is reduced (pass 1) and turned into dlogits (pass 2) out of one buffer, the
// bulk copies of the next rows into the others are already in flight, so that DRAM sees each row read once
// and written once and, but for a block's first row, the consumers find their row in shared memory.
// Longer rows are cut into kCluster contiguous slices, one per block of a cluster: every block runs the
// pipeline on its slice (its own producer thread, its own two slice buffers), and once per row the blocks
// exchange their partial partition sums through distributed shared memory (one asynchronous 16-byte store
// per peer, which completes on the peer's mbarrier), after which every block holds the same row total and
// finishes its slice on its own.
//
// Work distribution.  A block that holds whole rows (kCluster == 1) takes its rows from a counter in the
// workspace, one at a time, in row-major order of all B*T rows: a padded row is zero-filled on the spot by
// the producer thread, a valid row goes through the pipeline.  (The SMs do not see the same memory
// bandwidth and latency, so a static deal leaves the slowest block 10 to 20% behind the median.)  Results
// do not depend on which block gets which row: a row's outputs are a function of the row alone, and the
// policy loss is not summed per block: every row's term goes to the per-token area of the workspace, and
// the block that finishes last adds all of them in a fixed order.  Clusters take their rows statically
// (cluster c the valid rows c, c + G, ...): their rows are long and uniform.
//
// Pipeline of one block: a producer thread loads slice i+1 into the other buffer while the consumers work
// on slice i (it also requests each row's token id, old log-prob and advantage two rows ahead, so that it
// never waits for them); the consumers write the bf16 gradient over the logits in the buffer and hand it
// back; the producer drains it to global memory with one bulk store and refills it.  Waits are bounded
// (RowArgs::wait_limit_ns); if one runs out the thread flags RLHF_ERR_TIMEOUT, stops waiting and lets the
// block drain.  The tensor-memory columns are released by the warp that took them, after all consumers
// have passed a block barrier at the end of the kernel.
//
// kDistill: the row's loss is distillation from up to 256 teacher entries instead of an objective of one generated
// token.  Three more warps serve it.  Two target warps, in turn, turn the entries of a row into weights before the row has
// landed, then take the logits of those entries out of the buffer (they become -inf, as the generated token's does
// above, so that the sum over the other entries -- the student's mass outside the teacher's entries -- comes without
// cancellation).  The consumers' two passes are as above, with one factor for all entries that are not the teacher's.
// The patch warp then writes the gradients of the teacher's entries into the finished buffer and forms the row's loss,
// while the consumers are on the next row; the producer drains the buffer when it is done.
#pragma once
#include "kernels_ring.cuh"

namespace rlhf {

constexpr long long kTailPads = 2;      // padded rows of a cluster that are zero-filled after its last load

// What the producer publishes for each row before it arms the row's "landed" barrier.
struct RowInfo {
    long long flat;         // b*T + t
    long long dl_offset;    // element offset of the dlogits row
    int y;                  // generated token (0 if it was out of range)
    int bad_id;
    RowScalars sc;
    unsigned mis;           // bytes between the 16-byte boundary below the row's first logit and that logit
    unsigned pad;
};

// Block-wide total of the partial sums without the generated token's term, as consumer_reduce but with log2(NW) cross-warp steps.
template <int NW>
__device__ __forceinline__ Acc creg_reduce_rest(const Acc& a, float2* s_part, int warp, int lane)
{
    float M = a.M;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    float s = a.s * ex2(a.M - M);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) s_part[warp] = make_float2(M, s);
    asm volatile("bar.sync 1, %0;" ::"n"(NW * 32) : "memory");
    constexpr int kTop = NW > 16 ? 16 : (NW > 8 ? 8 : 4);
    const float2 pw = lane < NW ? s_part[lane] : make_float2(kFloorM, 0.f);
    float Mt = pw.x;
#pragma unroll
    for (int o = kTop; o > 0; o >>= 1) Mt = fmaxf(Mt, __shfl_xor_sync(0xffffffffu, Mt, o));
    float st = pw.y * ex2(pw.x - Mt);
#pragma unroll
    for (int o = kTop; o > 0; o >>= 1) st += __shfl_xor_sync(0xffffffffu, st, o);
    // lanes >= 2*kTop did not take part; everyone takes lane 0's result
    Mt = __shfl_sync(0xffffffffu, Mt, 0);
    st = __shfl_sync(0xffffffffu, st, 0);
    return Acc{Mt, st, 0.f};
}

// The same sum and another's term against the larger of the two references.
__device__ __forceinline__ Acc creg_add_label(const Acc& rest, const LabelInfo& li)
{
    Acc tot;
    tot.M = fmaxf(rest.M, li.M);
    tot.s = rest.s * ex2(rest.M - tot.M);
    tot.ey = li.ey * ex2(li.M - tot.M);
    return tot;
}

template <int NW>
__device__ __forceinline__ Acc creg_reduce(const Acc& a, float2* s_part, const LabelInfo* s_lab, int warp, int lane)
{
    const Acc rest = creg_reduce_rest<NW>(a, s_part, warp, lane);
    return creg_add_label(rest, *s_lab);
}

#ifndef RLHF_CREG_REGVECS_ONLY
#define RLHF_CREG_REGVECS_ONLY 8
#endif
constexpr int kRegVecsOnly = RLHF_CREG_REGVECS_ONLY;        // vectors per consumer thread when the registers hold all of a thread's exponentials
constexpr int kRegVecsTmem = 4;        // vectors per consumer thread kept in registers when the rest goes to tensor memory
constexpr int kTmemVecs = 16;          // at most so many vectors per consumer thread in tensor memory
constexpr int kCregZeroBytes = 16384;  // zeroed buffer that feeds the bulk zero-fill of padded rows
#ifndef RLHF_CREG_PIECE
#define RLHF_CREG_PIECE 16384
#endif

constexpr int kDistillMax = 256;       // teacher entries per row
constexpr int kDistillZeroBytes = 4096;
constexpr int kDistillSets = 4;         // rows whose entries are held (a power of two)
constexpr int kDistillRows = 8;         // rows announced to the target warps (a power of two)
constexpr int kDistillPlain = 0, kDistillNormalised = 1, kDistillTail = 2;

struct DistillArgs {
    const int* ids;          // teacher entries of row (b,t): [b*stride_b + t*stride_t + k], k < K; < 0 = unused
    const float* logprobs;
    long long stride_b, stride_t;
    int K, mode;
    float tau, scale;        // temperature, log2(e) / temperature
};

// A row, as it is announced to the target warps when the producer learns of it, two rows before it is loaded.
struct TargetRow {
    long long entries;       // element offset of its teacher entries, or -1: no more rows
    unsigned eoff;           // entries of its first vector that precede it
};

// What the target warp knows of a row's teacher entries.
struct TargetInfo {
    double H;                // sum p log p over the entries
    float P, p0, W;          // sum p; mass outside them (tail mode); P + p0
    float pr[4];             // sum p over the entries of each block's slice
};

// A row's sums.  x are the scaled logits, M the row's reference.  The mass outside the teacher's entries is kept against a
// reference of its own too: against M it may be far below the range of fp32, and the tail term takes its logarithm and its inverse.
struct DistillTotals {
    float M, s, ey;          // sums of 2^(x - M) over the entries that are not the teacher's and over those that are
    float zy;                // sum_k p_k (x_k - M)
    float Mo, so;            // sum of 2^(x - Mo) over the entries that are not the teacher's: at least 1/2, or 0 if there is none
};

// Whether a row's loss has the tail term: the teacher has mass outside its entries, and so has the student.  Loss, factor and the
// entries' gradients all ask here, so that the gradient is that of the loss.
__device__ __forceinline__ bool distill_has_tail(const TargetInfo& ti, float so) { return ti.p0 > 0.f && so > 0.f; }

// Weight of q_v in the gradient of a teacher's entry, d loss / d z_v = (weight * q_v - p_v) / tau: the weights of the terms that
// the loss has.
__device__ __forceinline__ float distill_weight(const TargetInfo& ti, float so) { return distill_has_tail(ti, so) ? ti.W : ti.P; }

// The gradient of a row's entries that are not the teacher's, d loss / d z_v = factor * 2^(x_v - M) / sum / tau: P q_v, and
// (W - p0 / q0) q_v = (W q0 - p0) q_v / q0 where there is a tail term, q0 the student's mass outside.  There M and sum are those
// of the mass outside alone, so that neither 1 / q0 nor q_v leaves the range of fp32.
struct DistillOutside {
    float factor, M, sum;
};
__device__ __forceinline__ DistillOutside distill_outside(const TargetInfo& ti, const DistillTotals& t, float q0)
{
    if (distill_has_tail(ti, t.so)) return DistillOutside{fmaf(ti.W, q0, -ti.p0), t.Mo, t.so};
    return DistillOutside{ti.P, t.M, t.s + t.ey};
}

// Loss of a row.  The logarithm of the mass outside is taken of s while that is in range: s and the sum s + ey share the error of
// the ex2 (2^-22) that brought s to the row's reference, and where most of the mass is outside it cancels (row losses at 8 x 64
// rows of 50272, tail mode: 1.5e-7 off, 2.5e-7 with so throughout).
__device__ __forceinline__ double distill_loss(const TargetInfo& ti, const DistillTotals& t)
{
    constexpr double ln2 = 0.6931471805599453;
    const double l2 = log2_split(t.s + t.ey);
    double L = ti.H - ln2 * ((double)t.zy - (double)ti.P * l2);
    if (distill_has_tail(ti, t.so)) {
        const double lo = t.s > 1e-20f ? log2_split(t.s) : log2_split(t.so) + ((double)t.Mo - (double)t.M);
        L += (double)ti.p0 * ln2 * (log2_split(ti.p0) - (lo - l2));
    }
    return L;
}

struct CregArgs {
    RowArgs row;
    unsigned row_bytes;      // 2*V, a multiple of 16
    unsigned slice_vecs;     // vectors per block of a cluster: ceil(row vectors / cluster size)
    unsigned buf_stride;     // bytes between the two slice buffers: a whole number of vectors per consumer thread
    unsigned tmem_cols;      // tensor-memory columns to take: 0, or a power of two from 32 to 512
    int n_buf;               // slice buffers per block: 2 or 3
    unsigned* row_counter;   // workspace word, zero between calls: next row to hand out (kCluster == 1)
    DistillArgs distill;     // kDistill
};

// A slice buffer holds the same number of vectors for every consumer thread; the vectors past the end of the
// slice are set to -inf once and never written again, so that the loops over a thread's vectors need no
// per-thread bound.
inline size_t creg_buf_stride(unsigned slice_vecs, int consumer_warps)
{
    const size_t per_round = (size_t)consumer_warps * 32;
    return (slice_vecs + per_round - 1) / per_round * per_round * 16;
}
constexpr int kCregMaxBufs = 3;
// K: teacher entries per row (0: not distillation), for each of which a set holds position, weight and logit.
inline int distill_pad(int K) { return (K + 31) / 32 * 32; }
inline size_t creg_smem_bytes(unsigned slice_vecs, int consumer_warps, int n_buf, int K = 0)
{
    return (size_t)n_buf * creg_buf_stride(slice_vecs, consumer_warps) + 12 * (size_t)distill_pad(K) * kDistillSets +
           (K > 0 ? kDistillZeroBytes : kCregZeroBytes) + 64;
}
// Columns of tensor memory that a block needs for slices of `slice_vecs` vectors: each warp stores 8 columns per
// vector beyond the first kRegVecsTmem; warps w, w+4, w+8, ... share 32 lanes and take consecutive column ranges.
inline unsigned creg_tmem_cols(unsigned slice_vecs, int consumer_warps)
{
    const unsigned per_round = (unsigned)consumer_warps * 32;
    const unsigned nj = (slice_vecs + per_round - 1) / per_round;
    if (nj <= (unsigned)kRegVecsOnly) return 0;
    const unsigned need = (nj - kRegVecsTmem) * 8 * (((unsigned)consumer_warps + 3) / 4);
    unsigned cols = 32;
    while (cols < need) cols *= 2;
    return cols;
}

// ---------------------------------------------------------------- cluster helpers
__device__ __forceinline__ uint32_t cluster_ctarank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Address, in the cluster's shared window, of this block's shared address `addr` in block `rank`.
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// 16 bytes into a peer's shared memory; the peer's mbarrier receives 16 transaction bytes when they are visible.
__device__ __forceinline__ void remote_store_v4(uint32_t remote_addr, const float4& v, uint32_t remote_bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(remote_addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(remote_bar) : "memory");
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same barrier for code in which the warps are no longer whole (the producer warp has one live lane).
__device__ __forceinline__ void cluster_sync_unaligned()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait for a phase that peers of the cluster complete.
__device__ __noinline__ bool mbar_wait_cluster_slow(uint32_t bar, uint32_t parity, unsigned* status,
                                                    unsigned long long limit_ns)
{
    const unsigned long long t0 = global_timer_ns();
    for (;;) {
        for (int i = 0; i < 128; ++i)
            if (mbar_try_wait_cluster(bar, parity)) return true;
        if (global_timer_ns() - t0 > limit_ns) {
            atomicOr(status, kErrTimeout);
            return false;
        }
    }
}

// Entry j of a vector replaced by -inf.
template <bool kF16>
__device__ __forceinline__ uint4 mask_vec_entry(const uint4& q, int j)
{
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i == j)
            w[i >> 1] = (i & 1) ? ((w[i >> 1] & 0x0000ffffu) | (El<kF16>::kNegInf << 16)) : ((w[i >> 1] & 0xffff0000u) | El<kF16>::kNegInf);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---------------------------------------------------------------- tensor memory as a scratch pad
// One warp takes `cols` columns (a power of two >= 32) for the block and writes their base address to shared memory.
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 8 values per thread: lane (of the warp's 32) x 8 consecutive columns.  Whole warp.
__device__ __forceinline__ void tmem_store8(uint32_t taddr, const float2 (&v)[4])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(__float_as_uint(v[0].x)), "r"(__float_as_uint(v[0].y)), "r"(__float_as_uint(v[1].x)),
                   "r"(__float_as_uint(v[1].y)), "r"(__float_as_uint(v[2].x)), "r"(__float_as_uint(v[2].y)),
                   "r"(__float_as_uint(v[3].x)), "r"(__float_as_uint(v[3].y)) : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t taddr, float2 (&v)[4])
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
#pragma unroll
    for (int h = 0; h < 4; ++h) v[h] = make_float2(__uint_as_float(r[2 * h]), __uint_as_float(r[2 * h + 1]));
}
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- what the target warps of the two on-chip-exponentials kernels do with a row's teacher entries (whole warp; lane l has
// the entries l, l + 32, ...)
constexpr int kPer = kDistillMax / 32;                       // entries per lane

// Weights pk, positions in this block's slice of the row (or -1), sum of the weights P, sum of p log p H, and the weights'
// sums over the slices of the cluster's blocks.  eoff: entries of the slice's first vector that precede the row.
template <int kCluster>
__device__ __forceinline__ void distill_weights(const RowArgs& p, const DistillArgs& dt, long long entries, uint32_t eoff,
                                                uint32_t v0, uint32_t nvec, uint32_t slice_vecs, uint32_t crank, int lane,
                                                int (&pos)[kPer], float (&pk)[kPer], double& P, double& H, float (&pr)[kCluster])
{
    float lt[kPer];
    bool bad = false;
    float lmax = kFloorM;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int k = lane + 32 * j;
        pos[j] = -1;
        lt[j] = __uint_as_float(0xff800000u);
        if (32 * j < dt.K && k < dt.K) {
            pos[j] = __ldg(dt.ids + entries + k);
            lt[j] = __ldg(dt.logprobs + entries + k);
            bad |= pos[j] < -1 || pos[j] >= p.V;
            if (pos[j] < 0 || pos[j] >= p.V) { pos[j] = -1; lt[j] = __uint_as_float(0xff800000u); }
            lmax = fmaxf(lmax, lt[j]);
        }
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0 && crank == 0) atomicOr(p.status, kErrIdRange);
    P = 0.0;
    if (dt.mode == kDistillNormalised) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lmax = fmaxf(lmax, __shfl_xor_sync(0xffffffffu, lmax, o));
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        pk[j] = 0.f;
        if (32 * j >= dt.K) continue;
        // tail: 1 - sum p is what the mass outside is worth, so the sum is formed of terms in double precision
        if (dt.mode == kDistillTail) { const double e = exp((double)lt[j]); P += e; pk[j] = (float)e; }
        else { pk[j] = expf(dt.mode == kDistillNormalised ? lt[j] - lmax : lt[j]); P += (double)pk[j]; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) P += __shfl_xor_sync(0xffffffffu, P, o);
    if (dt.mode == kDistillNormalised) {
        const float inv = P > 0.0 ? (float)(1.0 / P) : (P == P ? 0.f : (float)P), lse = lmax + (float)log(P);
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (32 * j < dt.K) { pk[j] *= inv; lt[j] -= lse; }
        P = P > 0.0 ? 1.0 : (P == P ? 0.0 : P);
    }
    H = 0.0;
#pragma unroll
    for (int c = 0; c < kCluster; ++c) pr[c] = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (32 * j >= dt.K) continue;
        if (!(pk[j] == 0.f)) H += (double)pk[j] * (double)lt[j];
        const uint32_t v = pos[j] < 0 ? 0xffffffffu : (eoff + (uint32_t)pos[j]) >> 3;
#pragma unroll
        for (int c = 0; c < kCluster; ++c)
            if (v - (uint32_t)c * slice_vecs < slice_vecs) pr[c] += pk[j];
        // position in this block's buffer, or -1
        pos[j] = v - v0 < nvec ? (int)(eoff + (uint32_t)pos[j] - v0 * 8u) : -1;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        H += __shfl_xor_sync(0xffffffffu, H, o);
#pragma unroll
        for (int c = 0; c < kCluster; ++c) pr[c] += __shfl_xor_sync(0xffffffffu, pr[c], o);
    }
}

// The first of several equal entries takes the weight of all, added in the order of the list; the others are dropped.
__device__ __forceinline__ void distill_merge(int K, int Kpad, int lane, int* tp, float* tw, int (&pos)[kPer], float (&pk)[kPer])
{
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int k = lane + 32 * j, mine = pos[j];
        if (mine < 0) continue;
        for (int o = 0; o < k; ++o)
            if (tp[o] == mine) { pos[j] = -1; break; }
        if (pos[j] < 0) { pk[j] = 0.f; continue; }
        for (int o = k + 1; o < K; ++o)
            if (tp[o] == mine) pk[j] += tw[o];
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (32 * j < Kpad) { tp[lane + 32 * j] = pos[j]; tw[lane + 32 * j] = pk[j]; }
}

// Sums over the slice's entries against their own largest exponent, and what the consumers and the patch warp need.
template <int kCluster>
__device__ __forceinline__ void distill_publish(const DistillArgs& dt, float xscale, uint32_t crank, int lane, const int (&pos)[kPer],
                                                const float (&pk)[kPer], const float (&z)[kPer], double P, double H,
                                                const float (&pr)[kCluster], TargetInfo& target, LabelInfo& lab)
{
    float Mt = kFloorM;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (32 * j < dt.K && pos[j] >= 0) Mt = fmaxf(Mt, z[j] * xscale);
    // (the largest by the warp-wide integer maximum: the bits of a float, negative ones complemented, order as the floats do)
    const int bits = __float_as_int(Mt), top = __reduce_max_sync(0xffffffffu, bits ^ ((bits >> 31) & 0x7fffffff));
    Mt = __int_as_float(top ^ ((top >> 31) & 0x7fffffff));
    float ey = 0.f, zy = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (32 * j < dt.K && pos[j] >= 0) {
            const float x = fmaf(z[j], xscale, -Mt);
            ey += ex2(x);
            if (!(pk[j] == 0.f)) zy = fmaf(pk[j], x, zy);
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        ey += __shfl_xor_sync(0xffffffffu, ey, o);
        zy += __shfl_xor_sync(0xffffffffu, zy, o);
    }
    if (lane == 0) {
        TargetInfo ti;
        ti.H = H;
        ti.P = (float)P;
        ti.p0 = dt.mode == kDistillTail ? (float)(1.0 - P > 0.0 ? 1.0 - P : 0.0) : 0.f;
        ti.W = dt.mode == kDistillTail ? (float)(P > 1.0 ? P : 1.0) : (float)P;
        if (!(P == P)) ti.W = ti.P;
        for (int c = 0; c < 4; ++c) ti.pr[c] = c < kCluster ? pr[c < kCluster ? c : 0] : 0.f;
        target = ti;
        lab = LabelInfo{zy, ey, Mt, ti.pr[crank]};
    }
}

// The same for few entries (kDistillFew at most), with loops that are not unrolled and entries that stay in shared memory.
// With a copy of every step per entry of a lane, most of them jumped over, the helping warps' code drives the consumers' out of
// the instruction cache: at V = 32000, K = 64 the warps waited for instructions 3.5 of 13.5 cycles per issue.  With many entries
// the unrolled steps are faster.  Rolled / unrolled, us, bf16, plain mode:
//     K                          64         96        128        160        256
//     16 x 512 rows of 32000   173 / 216  185 / 217  194 / 193  220 / 194  267 / 198
//     16 x 256 rows of 50272   146 / 145  148 / 145  152 / 146  158 / 146  176 / 148
//     16 x 256 rows of 80000   242 / 267  250 / 269  261 / 267  275 / 267  308 / 270
constexpr int kDistillFew = 96;

struct EntrySet {
    int* pos;                // position in the block's slice, or -1
    float* p;                // weight
    float* z;                // logit (log-prob until the row has landed)
    int K;
};

// Weights, positions, the sums of p and of p log p, and the weights' sums over the slices of the cluster's blocks.
// eoff: entries of the slice's first vector that precede the row.
template <int kCluster>
__device__ __forceinline__ void distill_weights_few(const RowArgs& p, const DistillArgs& dt, long long entries, uint32_t eoff,
                                                uint32_t v0, uint32_t nvec, uint32_t slice_vecs, uint32_t crank, int lane,
                                                const EntrySet& es, double& P, double& H, float (&pr)[kCluster])
{
    bool bad = false;
    float lmax = kFloorM;
#pragma unroll 2
    for (int k = lane; k < es.K; k += 32) {
        int id = __ldg(dt.ids + entries + k);
        float lt = __ldg(dt.logprobs + entries + k);
        bad |= id < -1 || id >= p.V;
        if (id < 0 || id >= p.V) { id = -1; lt = __uint_as_float(0xff800000u); }
        lmax = fmaxf(lmax, lt);
        es.pos[k] = id;
        es.z[k] = lt;
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0 && crank == 0) atomicOr(p.status, kErrIdRange);
    if (dt.mode == kDistillNormalised) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lmax = fmaxf(lmax, __shfl_xor_sync(0xffffffffu, lmax, o));
    } else {
        lmax = 0.f;
    }
    P = 0.0;
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32) {
        // tail: 1 - sum p is what the mass outside is worth, so the sum is formed of terms in double precision
        float e;
        if (dt.mode == kDistillTail) { const double x = exp((double)es.z[k]); P += x; e = (float)x; }
        else { e = expf(es.z[k] - lmax); P += (double)e; }
        es.p[k] = e;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) P += __shfl_xor_sync(0xffffffffu, P, o);
    float scale = 1.f, lse = 0.f;
    if (dt.mode == kDistillNormalised) {
        scale = P > 0.0 ? (float)(1.0 / P) : (P == P ? 0.f : (float)P);
        lse = lmax + (float)log(P);
        P = P > 0.0 ? 1.0 : (P == P ? 0.0 : P);
    }
    H = 0.0;
#pragma unroll
    for (int c = 0; c < kCluster; ++c) pr[c] = 0.f;
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32) {
        const float w = es.p[k] * scale;
        es.p[k] = w;
        if (!(w == 0.f)) H += (double)w * (double)(es.z[k] - lse);
        const int id = es.pos[k];
        const uint32_t v = id < 0 ? 0xffffffffu : (eoff + (uint32_t)id) >> 3;
#pragma unroll
        for (int c = 0; c < kCluster; ++c)
            if (v - (uint32_t)c * slice_vecs < slice_vecs) pr[c] += w;
        es.pos[k] = v - v0 < nvec ? (int)(eoff + (uint32_t)id - v0 * 8u) : -1;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        H += __shfl_xor_sync(0xffffffffu, H, o);
#pragma unroll
        for (int c = 0; c < kCluster; ++c) pr[c] += __shfl_xor_sync(0xffffffffu, pr[c], o);
    }
}

// Takes the entries' logits out of the row: they become -inf.  Every entry leaves its number in its place and looks whether it
// is still there: if not, the same entry is named twice.
template <bool kF16>
__device__ __forceinline__ bool distill_take_few(const EntrySet& es, uint16_t* row16, int lane)
{
    bool twice = false;
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) es.z[k] = El<kF16>::widen(row16[es.pos[k]]);
    __syncwarp();
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) row16[es.pos[k]] = (uint16_t)k;
    __syncwarp();
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) twice |= row16[es.pos[k]] != (uint16_t)k;
    __syncwarp();
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) row16[es.pos[k]] = (uint16_t)El<kF16>::kNegInf;
    __syncwarp();
    return twice;
}

// The first of several equal entries takes the weight of all, added in the order of the list; the others are dropped.
__device__ __noinline__ void distill_merge_few(const EntrySet es, int lane)
{
    __syncwarp();
    // a lane's new weights and positions wait until every lane has read the old ones: one entry per lane at a time
    for (int k0 = 0; k0 < es.K; k0 += 32) {
        const int k = k0 + lane, mine = k < es.K ? es.pos[k] : -1;
        bool later = false;
        float w = k < es.K ? es.p[k] : 0.f;
        if (mine >= 0) {
            for (int o = 0; o < k; ++o) later |= es.pos[o] == mine;
            for (int o = k + 1; o < es.K && !later; ++o)
                if (es.pos[o] == mine) w += es.p[o];
        }
        __syncwarp();
        if (mine >= 0 && !later) es.p[k] = w;                // (read by no entry before it, and dropped ones after it are not)
        __syncwarp();
    }
    for (int k0 = es.K - 1 - (es.K - 1) % 32; k0 >= 0; k0 -= 32) {
        const int k = k0 + lane, mine = k < es.K ? es.pos[k] : -1;
        bool later = false;
        if (mine >= 0)
            for (int o = 0; o < k; ++o) later |= es.pos[o] == mine;
        __syncwarp();
        if (later) { es.pos[k] = -1; es.p[k] = 0.f; }
        __syncwarp();
    }
}

// Sums over the slice's entries against their own largest exponent, and what the consumers and the patch warp need.
template <int kCluster>
__device__ __forceinline__ void distill_publish_few(const DistillArgs& dt, float xscale, uint32_t crank, int lane, const EntrySet& es,
                                                double P, double H, const float (&pr)[kCluster], TargetInfo& target, LabelInfo& lab)
{
    float Mt = kFloorM;
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) Mt = fmaxf(Mt, es.z[k] * xscale);
    // (the largest by the warp-wide integer maximum: the bits of a float, negative ones complemented, order as the floats do)
    const int bits = __float_as_int(Mt), top = __reduce_max_sync(0xffffffffu, bits ^ ((bits >> 31) & 0x7fffffff));
    Mt = __int_as_float(top ^ ((top >> 31) & 0x7fffffff));
    float ey = 0.f, zy = 0.f;
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) {
            const float x = fmaf(es.z[k], xscale, -Mt);
            ey += ex2(x);
            if (!(es.p[k] == 0.f)) zy = fmaf(es.p[k], x, zy);
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        ey += __shfl_xor_sync(0xffffffffu, ey, o);
        zy += __shfl_xor_sync(0xffffffffu, zy, o);
    }
    if (lane == 0) {
        target.H = H;
        target.P = (float)P;
        target.p0 = dt.mode == kDistillTail ? (float)(1.0 - P > 0.0 ? 1.0 - P : 0.0) : 0.f;
        target.W = !(P == P) ? (float)P : (dt.mode == kDistillTail ? (float)(P > 1.0 ? P : 1.0) : (float)P);
        float mine = pr[0];
#pragma unroll
        for (int c = 0; c < kCluster; ++c) {
            target.pr[c] = pr[c];
            if ((uint32_t)c == crank) mine = pr[c];
        }
        lab = LabelInfo{zy, ey, Mt, mine};
    }
}

// The gradients of the entries, as 16-bit patterns in the place of the weights.
template <bool kF16>
__device__ __forceinline__ void distill_values_few(const EntrySet& es, const DistillTotals& tot, const TargetInfo& ti, float xscale,
                                               float row_scale, int lane)
{
    const float l2 = log2f(tot.s + tot.ey), weight = distill_weight(ti, tot.so);
#pragma unroll 1
    for (int k = lane; k < es.K; k += 32)
        if (es.pos[k] >= 0) {
            const float q = ex2(fmaf(es.z[k], xscale, -tot.M) - l2);
            es.p[k] = __uint_as_float(El<kF16>::pack2(row_scale * fmaf(weight, q, -es.p[k]), 0.f) & 0xffffu);
        }
}

// The row's sums from those of the cluster's blocks, added in rank order: the same in every block.  xchg: (Mo, so, M, ey) of every
// block, M the reference of its entries, then their zy against that M.
template <int kCluster>
__device__ __forceinline__ void distill_cluster_totals(const float4* xchg, const TargetInfo& ti, Acc& rest, Acc& tot, float& zy)
{
    float Mo = kFloorM;
#pragma unroll
    for (int r = 0; r < kCluster; ++r) Mo = fmaxf(Mo, xchg[r].x);
    float so = 0.f, M = Mo;
#pragma unroll
    for (int r = 0; r < kCluster; ++r) {
        so = fmaf(xchg[r].y, ex2(xchg[r].x - Mo), so);
        M = fmaxf(M, xchg[r].z);
    }
    float ey = 0.f;
    zy = 0.f;
#pragma unroll
    for (int r = 0; r < kCluster; ++r) {
        ey = fmaf(xchg[r].w, ex2(xchg[r].z - M), ey);
        zy += fmaf(ti.pr[r], xchg[r].z - M, xchg[kCluster + r].x);
    }
    rest = Acc{Mo, so, 0.f};
    tot = Acc{M, so * ex2(Mo - M), ey};
}

// ---------------------------------------------------------------- the kernel
// kTmem: a thread's vectors beyond the first kRegVecsTmem keep their exponentials in tensor memory; otherwise a
// thread has at most kRegVecsOnly vectors and registers hold all of them.  kF16: logits and gradient are IEEE
// binary16 instead of bf16.  kAny (single blocks only): rows, of logits and dlogits alike and with the same offset
// from a 16-byte boundary, may start at any even address and have any length; the aligned span around a row is
// loaded, the entries of its first and last vector that belong to neighbouring rows are turned into -inf in the
// buffer before the first pass, and only the row's own bytes are stored: whole vectors by bulk store, the ragged
// ends by 2-byte stores.
// kDistill: see the head of the file.
template <int NW, int kCluster, bool kTmem, bool kF16, bool kAny = false, bool kDistill = false>
__global__ void __launch_bounds__(NW * 32 + (kDistill ? 128 : 32), 1) loss_creg_kernel(CregArgs ca)
{
    static_assert(!kAny || kCluster == 1, "rows off 16-byte boundaries are not split over a cluster");
    constexpr int kRegVecs = kTmem ? kRegVecsTmem : kRegVecsOnly;
    constexpr int kCons = NW * 32;
    constexpr int kThreads = kCons + (kDistill ? 128 : 32);
    constexpr int kZeroBytesHere = kDistill ? kDistillZeroBytes : kCregZeroBytes;
    constexpr uint32_t kPiece = RLHF_CREG_PIECE;  // size of one bulk copy
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long s_cnt[33];
    __shared__ float2 s_part[2][32];
    __shared__ __align__(16) float s_sum[2][(NW + 3) / 4 * 4];
    __shared__ LabelInfo s_lab[2];
    __shared__ RowInfo s_row[kCregMaxBufs];
    __shared__ double s_dbl[32];
    __shared__ double s_loss[2];
    __shared__ int s_last;
    // per row parity: (M, s, ey, zy) of every block of the cluster; kDistill: (Mo, so, M, ey) and zy, M the entries' reference
    __shared__ __align__(16) float4 s_xchg[2][kDistill ? 2 * kCluster : kCluster];
    __shared__ __align__(8) unsigned long long s_xbar[2];
    static_assert(NW <= 16, "the final sums take 16 doubles of scratch each");
    // rows that may be announced and not yet read by their target warp: those in the buffers, the row being taken, two ahead
    static_assert(kCregMaxBufs + 3 <= kDistillRows, "an announcement must not replace one that has not been read");
    static_assert(kCregMaxBufs * 16 <= 64, "the mbarriers of the buffers take the 64 bytes after the zero buffer");
    __shared__ uint32_t s_tmem_base;
    // kDistill: barriers ready / patched of every buffer, announced of every row that the target warps learn of, told / spare
    // / totals of every set of entries, and what target warps, consumers and patch warp hand on
    constexpr int kBufsHere = kDistill ? kCregMaxBufs : 1, kSetsHere = kDistill ? kDistillSets : 1;
    __shared__ __align__(8) unsigned long long s_dbar[kDistill ? 2 * kBufsHere + kDistillRows + 3 * kDistillSets : 1];
    __shared__ TargetRow s_trow[kDistill ? kDistillRows : 1];
    __shared__ TargetInfo s_target[kSetsHere];
    __shared__ LabelInfo s_tlab[kSetsHere];
    __shared__ DistillTotals s_total[kSetsHere];

    const RowArgs& p = ca.row;
    const DistillArgs& dt = ca.distill;
    const float xscale = kDistill ? dt.scale : kLog2e;       // logit -> base-2 exponent
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int NB = ca.n_buf;
    const uint32_t crank = kCluster > 1 ? cluster_ctarank() : 0u;
    const long long cid = blockIdx.x / kCluster;             // this block's cluster
    const long long G = gridDim.x / kCluster;                // clusters in the grid
    const uint32_t row_vecs = kAny ? ca.slice_vecs : ca.row_bytes / 16u;   // kAny: the longest aligned span around a row
    const uint32_t v0 = min(row_vecs, crank * ca.slice_vecs);      // this block's slice of every row: vectors [v0, v0+nvec)
    const uint32_t nvec = min(row_vecs - v0, ca.slice_vecs);
    const uint32_t slice_off = v0 * 16u, slice_bytes = nvec * 16u;

    const uint32_t buf_addr = smem_u32(smem);
    unsigned char* zero_buf = smem + (size_t)NB * ca.buf_stride;
    const uint32_t bar_addr = smem_u32(zero_buf + kZeroBytesHere);
    auto landed = [&](int buf) { return bar_addr + 8u * buf; };
    auto computed = [&](int buf) { return bar_addr + 8u * (kCregMaxBufs + buf); };
    const uint32_t xbar_addr = smem_u32(s_xbar);
    const uint32_t dbar = smem_u32(s_dbar);
    auto ready = [&](int buf) { return dbar + 8u * buf; };                          // teacher entries taken out
    auto patched = [&](int buf) { return dbar + 8u * (kBufsHere + buf); };
    auto announced = [&](int i) { return dbar + 8u * (2 * kBufsHere + (i & (kDistillRows - 1))); };
    const uint32_t sbar = dbar + 8u * (2 * kBufsHere + kDistillRows);
    auto told = [&](int i) { return sbar + 8u * (i & (kDistillSets - 1)); };                          // the entries' sums are there
    auto totals = [&](int i) { return sbar + 8u * (kDistillSets + (i & (kDistillSets - 1))); };       // the row's are
    auto spare = [&](int i) { return sbar + 8u * (2 * kDistillSets + (i & (kDistillSets - 1))); };    // the set has been read
    auto set_phase = [&](int i) { return (uint32_t)(i / kDistillSets) & 1u; };
    const int Kpad = kDistill ? (dt.K + 31) / 32 * 32 : 0;
    // teacher entries of a row: position in the buffer (or -1), weight, logit
    auto t_pos = [&](int i) { return (int*)(zero_buf + kZeroBytesHere + 64) + 3 * (i & (kDistillSets - 1)) * Kpad; };
    auto t_p = [&](int i) { return (float*)t_pos(i) + Kpad; };
    auto t_z = [&](int i) { return (float*)t_pos(i) + 2 * Kpad; };
    const bool few = kDistill && dt.K <= kDistillFew;

    if (tid == 0) {
        for (int b = 0; b < NB; ++b) {
            mbar_init(landed(b), 1);
            mbar_init(computed(b), NW);
            if (kDistill) {
                mbar_init(ready(b), 1);
                mbar_init(patched(b), 1);
            }
        }
        for (int i = 0; kDistill && i < kDistillRows; ++i) mbar_init(announced(i), 1);
        for (int i = 0; kDistill && i < kDistillSets; ++i) {
            mbar_init(told(i), 1);
            mbar_init(totals(i), 1);
            mbar_init(spare(i), 1);
        }
        mbar_init(xbar_addr, 1);
        mbar_init(xbar_addr + 8u, 1);
        fence_mbar_init();
    }
    if (kTmem && warp == 0) tmem_alloc(smem_u32(&s_tmem_base), ca.tmem_cols);
    for (int i = tid; i < kZeroBytesHere / 16; i += kThreads) ((uint4*)zero_buf)[i] = make_uint4(0, 0, 0, 0);
    // the vectors of every buffer past the end of the slice: -inf, a term of 0 in every sum
    for (int b = 0; b < NB; ++b)
        for (uint32_t v = nvec + tid; v < ca.buf_stride / 16u; v += kThreads)
            ((uint4*)(smem + (size_t)b * ca.buf_stride))[v] = make_uint4(El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2);
    fence_async_smem();
    if (kTmem) tmem_fence_before_sync();
    __syncthreads();
    if (kTmem) tmem_fence_after_sync();
    if (kCluster > 1) cluster_sync_all();        // every peer's barriers exist before anyone signals them
    pdl_wait_prior_grid();                       // nothing above touches global memory
    pdl_release_next_grid();

    const long long N = block_count_valid(p.lengths, p.B, p.T, s_cnt, blockIdx.x == 0 ? p.status : nullptr);
    const long long D = p.seq_mean ? block_count_nonempty(p.lengths, p.B, s_cnt) : N;   // what the loss is a mean over
    const int n_mine = N > cid ? (int)((N - cid + G - 1) / G) : 0;   // rows of this cluster: cid, cid + G, ...

    bool aborted = false;

    if (warp == NW) {
        // ------------------------------------------------------------ producer
        if (lane == 0) {
            const long long total_rows = (long long)p.B * p.T;
            const long long n_pad = total_rows - N;
            const PadShare pads = kCluster > 1 ? pad_share(N, n_pad, G, cid) : PadShare{0, 0};   // static deal: padded rows of the cluster
            const long long pads_mine = pads.count;
            const long long pads_early = pads_mine > kTailPads ? pads_mine - kTailPads : 0;
            Cursor cur{0, 0}, pcur{0, 0};
            long long pads_done = 0;
            auto zero_fill_row = [&](int b, int t) {
                unsigned char* drow = (unsigned char*)(p.dlogits + (long long)b * p.dl_stride_b + (long long)t * p.dl_stride_t) + slice_off;
                uint32_t lo = 0, hi = slice_bytes;                   // [lo,hi): the part of the row made of whole 16-byte vectors
                if (kAny) {
                    const uint32_t mis = (uint32_t)((uintptr_t)drow & 15u);
                    lo = min(ca.row_bytes, (16u - mis) & 15u);
                    hi = max(lo, ca.row_bytes - ((mis + ca.row_bytes) & 15u));
                    for (uint32_t o = 0; o < lo; o += 2) *(uint16_t*)(drow + o) = 0;
                    for (uint32_t o = hi; o < ca.row_bytes; o += 2) *(uint16_t*)(drow + o) = 0;
                }
                for (uint32_t off = lo; off < hi; off += kZeroBytesHere)
                    bulk_store(drow + off, smem_u32(zero_buf), min((uint32_t)kZeroBytesHere, hi - off));
                bulk_commit();
            };
            auto zero_fill_next = [&]() {
                int b, t;
                if (!cursor_seek_padded(pcur, pads.start + pads_done, p.lengths, p.B, p.T, b, t)) return;
                zero_fill_row(b, t);
            };
            // Hands buffer i % NB, holding the finished gradient of this block's i-th slice, to the bulk-store
            // engine and waits until it has been read out of shared memory.
            auto drain = [&](int i) {
                const int buf = i % NB;
                mbar_wait(kDistill ? patched(buf) : computed(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
                if (aborted) return;
                const uint32_t srcb = buf_addr + (uint32_t)buf * ca.buf_stride;
                unsigned char* drow = (unsigned char*)(p.dlogits + s_row[buf].dl_offset) + slice_off;
                uint32_t mis = 0, lo = 0, hi = slice_bytes;          // row = span bytes [mis, mis + row_bytes); whole vectors [lo,hi)
                if (kAny) {
                    mis = (uint32_t)((uintptr_t)drow & 15u);
                    lo = (mis + 15u) & ~15u;
                    hi = (mis + ca.row_bytes) & ~15u;
                    if (hi < lo) hi = lo;
                    const unsigned char* sb = smem + (size_t)buf * ca.buf_stride;
                    for (uint32_t o = mis; o < min(lo, mis + ca.row_bytes); o += 2) *(uint16_t*)(drow - mis + o) = *(const uint16_t*)(sb + o);
                    for (uint32_t o = max(hi, mis); o < mis + ca.row_bytes; o += 2) *(uint16_t*)(drow - mis + o) = *(const uint16_t*)(sb + o);
                    fence_async_smem();                              // these reads, before the buffer is refilled by bulk copies
                }
                for (uint32_t off = lo; off < hi; off += kPiece)
                    bulk_store(drow - mis + off, srcb + off, min(kPiece, hi - off));
                bulk_commit();
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            };
            // The scalars of a row (token id, old log-prob, advantage) are requested two rows ahead of their use.
            struct Ahead {
                int b, t;
                long long y;
                RowScalars sc;
                bool ok;
            };
            long long k_ahead = cid;
            // dynamic deal: the next row of the row-major list of all rows, requested one call ahead of its use
            long long r_next = 0;
            if (kCluster == 1) r_next = (long long)atomicAdd(ca.row_counter, 1u);
            auto fetch = [&]() {
                Ahead a;
                a.ok = false;
                if (kCluster == 1) {
                    while (r_next < total_rows) {
                        const long long r = r_next;
                        r_next = (long long)atomicAdd(ca.row_counter, 1u);
                        a.b = (int)(r / p.T);
                        a.t = (int)(r % p.T);
                        if (a.t < clamp_len(__ldg(p.lengths + a.b), p.T)) { a.ok = true; break; }
                        zero_fill_row(a.b, a.t);                       // a padded row: nothing to read
                    }
                } else {
                    a.ok = k_ahead < N && cursor_seek_valid(cur, k_ahead, p.lengths, p.B, p.T, a.b, a.t);
                    k_ahead += G;
                }
                if (a.ok) {
                    const long long f = (long long)a.b * p.T + a.t;
                    a.y = kDistill ? 0 : __ldg(p.ids + (long long)a.b * p.ids_stride_b + a.t);
                    if (!kDistill) a.sc = load_row_scalars(p, a.b, a.t, f);
                }
                return a;
            };
            // the target warps learn of a row as soon as the producer does
            auto announce = [&](int j, const Ahead& a) {
                if (!kDistill) return;
                TargetRow tr{-1, 0u};
                if (a.ok) {
                    tr.entries = (long long)a.b * dt.stride_b + (long long)a.t * dt.stride_t;
                    if (kAny) tr.eoff = (unsigned)((uintptr_t)(p.logits + (long long)a.b * p.stride_b + (long long)a.t * p.stride_t) & 15u) >> 1;
                }
                s_trow[j & (kDistillRows - 1)] = tr;
                mbar_arrive(announced(j));
            };
            Ahead a0 = fetch(), a1 = fetch();
            announce(0, a0);
            announce(1, a1);
            int i = 0;
            for (; !aborted; ++i) {
                const Ahead a = a0;
                a0 = a1;
                a1 = fetch();
                announce(i + 2, a1);
                if (!a.ok) break;
                const unsigned char* row = (const unsigned char*)(p.logits + (long long)a.b * p.stride_b + (long long)a.t * p.stride_t) + slice_off;
                RowInfo ri;
                ri.flat = (long long)a.b * p.T + a.t;
                ri.dl_offset = (long long)a.b * p.dl_stride_b + (long long)a.t * p.dl_stride_t;
                ri.bad_id = (a.y < 0 || a.y >= p.V) ? 1 : 0;
                ri.y = ri.bad_id ? 0 : (int)a.y;
                if (!kDistill) ri.sc = a.sc;
                ri.mis = kAny ? (unsigned)((uintptr_t)row & 15u) : 0u;
                ri.pad = 0;
                if (ri.bad_id && crank == 0) atomicOr(p.status, kErrIdRange);
                const int buf = i % NB;
                if (i >= NB) drain(i - NB);                              // the buffer's previous slice goes out first
                if (aborted) break;
                s_row[buf] = ri;
                const uint32_t dst = buf_addr + (uint32_t)buf * ca.buf_stride;
                // kAny: the aligned span around the row (it stays inside the 16-byte blocks that hold the row's ends)
                const uint32_t load_bytes = kAny ? ((ri.mis + ca.row_bytes + 15u) & ~15u) : slice_bytes;
                mbar_arrive_expect_tx(landed(buf), load_bytes);          // release: publishes s_row[buf]
                for (uint32_t off = 0; off < load_bytes; off += kPiece)
                    bulk_load(dst + off, row - ri.mis + off, min(kPiece, load_bytes - off), landed(buf));
                if (kCluster > 1) {
                    const long long target = ((long long)(i + 1) * pads_early) / n_mine;
                    while (pads_done < target) { zero_fill_next(); ++pads_done; }
                }
            }
            while (pads_done < pads_mine) { zero_fill_next(); ++pads_done; }
            // no more rows: the consumers are told through the next buffer's row info
            if (!aborted) {
                const int buf = i % NB;
                if (i >= NB) drain(i - NB);
                if (!aborted) {
                    s_row[buf].flat = -1;
                    mbar_arrive_expect_tx(landed(buf), 0);
                }
            }
            for (int j = i + 1 >= NB ? i + 1 - NB : 0; j < i && !aborted; ++j) drain(j);
            bulk_wait_all();
            if (kCluster > 1) cluster_sync_unaligned();                 // no block leaves while a peer may still write to it
        }
        return;
    }

    if (kDistill && (warp == NW + 1 || warp == NW + 2)) {
        // ------------------------------------------------------------ target warps: one for every other row
        for (int i = warp - (NW + 1); !aborted; i += 2) {
            const int buf = i % NB;
            mbar_wait(announced(i), (uint32_t)(i / kDistillRows) & 1u, p.status, aborted, p.wait_limit_ns);
            aborted = __any_sync(0xffffffffu, aborted);
            if (aborted) break;
            const TargetRow tr = s_trow[i & (kDistillRows - 1)];
            if (tr.entries < 0) break;
            float pr[kCluster];
            double P, H;
            if (few) {
                const EntrySet es{t_pos(i), t_p(i), t_z(i), dt.K};
                // the set's previous row has been patched (nothing to wait for in the first turn)
                mbar_wait(spare(i), set_phase(i) ^ 1u, p.status, aborted, p.wait_limit_ns);
                aborted = __any_sync(0xffffffffu, aborted);
                if (aborted) break;
                distill_weights_few<kCluster>(p, dt, tr.entries, tr.eoff, v0, nvec, ca.slice_vecs, crank, lane, es, P, H, pr);
                mbar_wait(landed(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
                aborted = __any_sync(0xffffffffu, aborted);
                if (aborted) break;
                const bool again = distill_take_few<kF16>(es, (uint16_t*)(smem + (size_t)buf * ca.buf_stride), lane);
                if (lane == 0) mbar_arrive(ready(buf));
                if (__any_sync(0xffffffffu, again)) distill_merge_few(es, lane);
                distill_publish_few<kCluster>(dt, xscale, crank, lane, es, P, H, pr, s_target[i & (kDistillSets - 1)],
                                              s_tlab[i & (kDistillSets - 1)]);
                __syncwarp();
                if (lane == 0) mbar_arrive(told(i));
                continue;
            }
            int pos[kPer];
            float pk[kPer];
            distill_weights<kCluster>(p, dt, tr.entries, tr.eoff, v0, nvec, ca.slice_vecs, crank, lane, pos, pk, P, H, pr);
            // the logits leave the buffer.  Every entry leaves its number in its place and looks whether it is still
            // there: if not, the same entry is named twice.
            mbar_wait(landed(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
            // the set's previous row has been patched (nothing to wait for in the first turn)
            mbar_wait(spare(i), set_phase(i) ^ 1u, p.status, aborted, p.wait_limit_ns);
            aborted = __any_sync(0xffffffffu, aborted);
            if (aborted) break;
            uint16_t* row16 = (uint16_t*)(smem + (size_t)buf * ca.buf_stride);
            int* tp = t_pos(i);
            float *tw = t_p(i), *tz = t_z(i);
            float z[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                z[j] = 0.f;
                if (32 * j < dt.K && pos[j] >= 0) z[j] = El<kF16>::widen(row16[pos[j]]);
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (32 * j < dt.K && pos[j] >= 0) row16[pos[j]] = (uint16_t)(lane + 32 * j);
            __syncwarp();
            bool twice = false;
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (32 * j < dt.K && pos[j] >= 0) twice |= row16[pos[j]] != (uint16_t)(lane + 32 * j);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                if (32 * j >= dt.K) break;
                if (pos[j] >= 0) row16[pos[j]] = (uint16_t)El<kF16>::kNegInf;
                { tp[lane + 32 * j] = pos[j]; tw[lane + 32 * j] = pk[j]; tz[lane + 32 * j] = z[j]; }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(ready(buf));
            if (__any_sync(0xffffffffu, twice)) distill_merge(dt.K, Kpad, lane, tp, tw, pos, pk);
            distill_publish<kCluster>(dt, xscale, crank, lane, pos, pk, z, P, H, pr, s_target[i & (kDistillSets - 1)],
                                      s_tlab[i & (kDistillSets - 1)]);
            __syncwarp();
            if (lane == 0) mbar_arrive(told(i));
        }
        return;
    }

    if (kDistill && warp == NW + 3) {
        // ------------------------------------------------------------ patch warp
        const float row_scale = N > 0 ? p.grad_scale * dt.tau / (float)N : 0.f;
        for (int i = 0; !aborted; ++i) {
            const int buf = i % NB;
            mbar_wait(totals(i), set_phase(i), p.status, aborted, p.wait_limit_ns);
            aborted = __any_sync(0xffffffffu, aborted);
            if (aborted) break;
            const long long flat = s_row[buf].flat;
            if (flat < 0) break;
            // the gradients of the entries, while the consumers write the others
            const DistillTotals tot = s_total[i & (kDistillSets - 1)];
            const TargetInfo ti = s_target[i & (kDistillSets - 1)];
            if (few) {
                const EntrySet es{t_pos(i), t_p(i), t_z(i), dt.K};
                distill_values_few<kF16>(es, tot, ti, xscale, row_scale, lane);
                mbar_wait(computed(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
                aborted = __any_sync(0xffffffffu, aborted);
                if (aborted) break;
                uint16_t* row16 = (uint16_t*)(smem + (size_t)buf * ca.buf_stride);
#pragma unroll 1
                for (int k = lane; k < dt.K; k += 32)
                    if (es.pos[k] >= 0) row16[es.pos[k]] = (uint16_t)__float_as_uint(es.p[k]);
                __syncwarp();
                if (lane == 0) mbar_arrive(spare(i));                // the set has been read
            } else {
                const float l2 = log2f(tot.s + tot.ey), weight = distill_weight(ti, tot.so);
                int pos[kPer];
                uint32_t value[kPer];
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int k = lane + 32 * j;
                    pos[j] = -1;
                    value[j] = 0;
                    if (32 * j < dt.K && k < dt.K) pos[j] = t_pos(i)[k];
                    if (32 * j < dt.K && pos[j] >= 0) {
                        const float q = ex2(fmaf(t_z(i)[k], xscale, -tot.M) - l2);
                        value[j] = El<kF16>::pack2(row_scale * fmaf(weight, q, -t_p(i)[k]), 0.f) & 0xffffu;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(spare(i));                    // the set has been read
                mbar_wait(computed(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
                aborted = __any_sync(0xffffffffu, aborted);
                if (aborted) break;
                uint16_t* row16 = (uint16_t*)(smem + (size_t)buf * ca.buf_stride);
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (32 * j < dt.K && pos[j] >= 0) row16[pos[j]] = (uint16_t)value[j];
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(patched(buf));
                if (crank == 0) {
                    const float L = (float)((double)dt.tau * (double)dt.tau * distill_loss(ti, tot));
                    p.row_loss[flat] = L;
                    if (p.out_lp_new) p.out_lp_new[flat] = L;
                }
            }
        }
        __threadfence();
        asm volatile("bar.sync 2, %0;" ::"n"(kCons + 32) : "memory");   // the row losses are written
        return;
    }

    // ---------------------------------------------------------------- consumers
    const float scale_over_N = N > 0 ? p.grad_scale / (float)D : 0.f;
    const int cnt = (uint32_t)tid < nvec ? (int)((nvec - tid + kCons - 1) / kCons) : 0;   // this thread's vectors
    const int nj = (int)((nvec + kCons - 1) / kCons);              // vectors per thread, the -inf tail included
    const int nt = kTmem && nj > kRegVecs ? nj - kRegVecs : 0;     // of which in tensor memory (<= kTmemVecs)
    // this warp's window of tensor memory: its 32 lanes, 8 columns per vector
    const uint32_t tmem_addr = kTmem ? s_tmem_base + (((uint32_t)(warp & 3) * 32u) << 16) + (uint32_t)(warp >> 2) * (uint32_t)(nt * 8) : 0u;
    // the block's share of the value loss (thread 0 keeps the sum); it also zeroes the per-token policy terms of the
    // padded tokens, so that the final sum can run over all B*T entries
    {
        const double vf = consumer_sum_double<NW>(value_loss_slice(p, N, tid, kCons, true), s_dbl, warp, lane);
        if (tid == 0) s_loss[1] = vf;
    }

    for (int i = 0;; ++i) {
        const int buf = i % NB, par = i & 1;
        const uint32_t use = (uint32_t)(i >> 1) & 1u;                // of the exchange barrier, which alternates by row
        mbar_wait(landed(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
        aborted = __any_sync(0xffffffffu, aborted);                 // a warp gives up as a whole
        RowInfo ri = s_row[buf];
        if (aborted) { ri.y = 0; ri.bad_id = 1; ri.flat = 0; }      // stale row info: touch nothing
        if (ri.flat < 0) {                                           // the producer has no more rows (the same for every thread)
            if (kDistill && tid == 0) mbar_arrive(totals(i));        // tells the patch warp
            break;
        }
        if (kDistill) {
            mbar_wait(ready(buf), (uint32_t)(i / NB) & 1u, p.status, aborted, p.wait_limit_ns);
            aborted = __any_sync(0xffffffffu, aborted);
        }
        unsigned char* rowbuf = smem + (size_t)buf * ca.buf_stride;
        const uint4* src = (const uint4*)rowbuf + tid;

        // kAny: eoff entries of the buffer's first vector precede the row; they, the entries after the row's end in its
        // last vector and the vector after that (left from a longer span) are not the row's: their owners make them -inf
        const uint32_t eoff = kAny ? (ri.mis >> 1) : 0u;
        if (kAny) {
            const uint32_t end = eoff + (uint32_t)p.V;               // entry index, in the buffer, of the row's end
            const uint32_t last = (end - 1) >> 3, past = last + 1;   // vector of the last entry, and the one after it
            uint4* vecs = (uint4*)rowbuf;
            if (eoff != 0 && tid == 0) vecs[0] = mask_vec_outside<kF16>(vecs[0], (int)eoff, 8);
            if ((end & 7u) != 0 && (last % kCons) == (uint32_t)tid) vecs[last] = mask_vec_outside<kF16>(vecs[last], 0, (int)(end & 7u));
            if (past < nvec && (past % kCons) == (uint32_t)tid)
                vecs[past] = make_uint4(El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2, El<kF16>::kNegInf2);
        }
        // where the generated token sits: vector ylocal of this slice (if < nvec), entry yj
        const uint32_t ylocal = ((eoff + (uint32_t)ri.y) >> 3) - v0;
        const int yj = (int)((eoff + (uint32_t)ri.y) & 7u);
        const bool label_here = !kDistill && ylocal < nvec;
        const bool owner = label_here && (ylocal % kCons) == (uint32_t)tid;
        const int jy = owner ? (int)(ylocal / kCons) : -1;

        // The reference exponent: the scaled maximum of the slice's first vector, which every thread reads; the
        // generated token's entry is left out of it, because its owner is replacing that entry in the buffer.
        float Mref = kFloorM;
        if (nvec > 0) {
            uint4 q0 = *(const uint4*)rowbuf;
            if (kAny) q0 = mask_vec_outside<kF16>(q0, (int)eoff, 8);
            if (label_here && ylocal == 0) q0 = mask_vec_entry<kF16>(q0, yj);
            Mref = max8_scaled<kF16>(q0, xscale);
        }
        // The owner takes the generated token's logit out of the row (it becomes -inf, a term of 0), so that
        // the sums below are sums over the other entries and 1 - p_y comes without cancellation.
        float zy = 0.f, xy = kFloorM;
        if (owner) {
            uint16_t* slot = (uint16_t*)rowbuf + ((size_t)ylocal * 8 + yj);
            zy = El<kF16>::widen(*slot);
            *slot = (uint16_t)El<kF16>::kNegInf;
            xy = fmaxf(zy * kLog2e, kFloorM);
        }

        // ---- pass 1: the exponentials of this thread's vectors against the reference; the first kRegVecs
        // vectors' stay in registers, the others' go to tensor memory
        float2 e[kRegVecs][4];
        auto fill = [&](float negM) -> float {
            float2 acc0 = make_float2(0.f, 0.f), acc1 = make_float2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < kRegVecs; ++j) {
                if (j < nj) {
                    const uint4 q = src[(size_t)j * kCons];
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const float2 x = __ffma2_rn(El<kF16>::unpack2(w[h]), splat2(xscale), splat2(negM));
                        e[j][h] = make_float2(ex2(x.x), ex2(x.y));
                    }
                    acc0 = __fadd2_rn(acc0, e[j][0]);
                    acc1 = __fadd2_rn(acc1, e[j][1]);
                    acc0 = __fadd2_rn(acc0, e[j][2]);
                    acc1 = __fadd2_rn(acc1, e[j][3]);
                } else {
#pragma unroll
                    for (int h = 0; h < 4; ++h) e[j][h] = make_float2(0.f, 0.f);
                }
            }
#pragma unroll 2
            for (int j = 0; kTmem && j < nt; ++j) {
                const uint4 q = src[(size_t)(kRegVecs + j) * kCons];
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                float2 et[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float2 x = __ffma2_rn(El<kF16>::unpack2(w[h]), splat2(xscale), splat2(negM));
                    et[h] = make_float2(ex2(x.x), ex2(x.y));
                }
                tmem_store8(tmem_addr + (uint32_t)j * 8u, et);
                acc0 = __fadd2_rn(acc0, et[0]);
                acc1 = __fadd2_rn(acc1, et[1]);
                acc0 = __fadd2_rn(acc0, et[2]);
                acc1 = __fadd2_rn(acc1, et[3]);
            }
            return (acc0.x + acc0.y) + (acc1.x + acc1.y);
        };
        float M = Mref, vs = 0.f;
#pragma unroll 1
        for (int attempt = 0;; ++attempt) {
            vs = fill(-M);
            // in range: every term at most 2^64 against the reference, the generated token's included
            const bool in_range = vs <= 1.8446744e19f && M > kFloorM && !(xy - M > kRebase);
            const bool redo = attempt == 0 && !in_range && (cnt > 0 || owner);
            // the tensor-memory stores are warp-wide: if any lane has to redo its share, the whole warp does
            if (!__any_sync(0xffffffffu, redo)) break;
            if (redo) {
                // a reference of this thread's own: its largest scaled entry
                float m = xy;
                for (int j = 0; j < nj; ++j) m = fmaxf(m, max8_scaled<kF16>(src[(size_t)j * kCons], xscale));
                M = m;
            }
        }
        if (cnt == 0 && !owner) { M = Mref; vs = 0.f; }
        const bool diverged = M != Mref;
        const int ts = i & (kDistillSets - 1);                       // kDistill: the row's set of entries
        if (kDistill) {
            mbar_wait(told(i), set_phase(i), p.status, aborted, p.wait_limit_ns);
            aborted = __any_sync(0xffffffffu, aborted);
        }

        if (!kDistill && (label_here ? owner : tid == 0))
            s_lab[par] = label_here ? LabelInfo{zy, ex2(fmaf(zy, kLog2e, -M)), M, 0.f} : LabelInfo{0.f, 0.f, kFloorM, 0.f};
        float ws = vs;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
        if (lane == 0) s_sum[par][warp] = ws;
        Acc tot, rest;                                               // kDistill: rest is the sum outside, against its own reference
        if (!consumer_barrier_or<NW>(diverged || aborted)) {
            tot.M = Mref;
            tot.s = sum_warp_sums<NW>(s_sum[par]);
            if (kDistill) rest = Acc{Mref, tot.s, 0.f};
            else tot.ey = s_lab[par].ey;
        } else {
            // a wait that ran out somewhere in the block ends the block's work here, for all its threads alike
            if (consumer_barrier_or<NW>(aborted)) { aborted = true; break; }
            if (kDistill) rest = creg_reduce_rest<NW>(Acc{M, vs, 0.f}, s_part[par], warp, lane);
            else tot = creg_reduce<NW>(Acc{M, vs, 0.f}, s_part[par], &s_lab[par], warp, lane);
        }
        float zy_row = kDistill ? 0.f : s_lab[par].zy;               // the generated token's logit; kDistill: DistillTotals::zy
        if (kDistill && kCluster == 1) {
            const LabelInfo li = s_tlab[ts];
            tot = creg_add_label(rest, li);
            zy_row = fmaf(li.pad, li.M - tot.M, li.zy);
        }

        if (kCluster > 1) {
            // every block of the cluster sends its slice's sums to every block, itself included
            if (tid == 0) {
                mbar_arrive_expect_tx(xbar_addr + 8u * par, (kDistill ? 32u : 16u) * kCluster);
                const LabelInfo li = kDistill ? s_tlab[ts] : LabelInfo{};
                const float4 mine = kDistill ? make_float4(rest.M, rest.s, li.M, li.ey) : make_float4(tot.M, tot.s, tot.ey, zy_row);
                const uint32_t slot = smem_u32(&s_xchg[par][crank]);
#pragma unroll
                for (int r = 0; r < kCluster; ++r) {
                    remote_store_v4(map_to_rank(slot, (uint32_t)r), mine, map_to_rank(xbar_addr + 8u * par, (uint32_t)r));
                    if (kDistill)
                        remote_store_v4(map_to_rank(slot + 16u * kCluster, (uint32_t)r), make_float4(li.zy, 0.f, 0.f, 0.f),
                                        map_to_rank(xbar_addr + 8u * par, (uint32_t)r));
                }
            }
            if (!aborted && !mbar_try_wait_cluster(xbar_addr + 8u * par, use))
                if (!mbar_wait_cluster_slow(xbar_addr + 8u * par, use, p.status, p.wait_limit_ns)) aborted = true;
            aborted = __any_sync(0xffffffffu, aborted);
            if (kDistill) {
                distill_cluster_totals<kCluster>(s_xchg[par], s_target[ts], rest, tot, zy_row);
            } else {
                float Mx = kFloorM;
#pragma unroll
                for (int r = 0; r < kCluster; ++r) Mx = fmaxf(Mx, s_xchg[par][r].x);
                float sx = 0.f, eyx = 0.f, zx = 0.f;
#pragma unroll
                for (int r = 0; r < kCluster; ++r) {               // in rank order: the same total in every block
                    const float4 part = s_xchg[par][r];
                    const float sc = ex2(part.x - Mx);
                    sx = fmaf(part.y, sc, sx);
                    eyx = fmaf(part.z, sc, eyx);
                    zx += part.w;
                }
                tot = Acc{Mx, sx, eyx};
                zy_row = zx;
            }
        }
        RowResult r = row_finish_fast(tot, zy_row);

        float loss = 0.f, kl = 0.f, g = 0.f;
        float den_M = tot.M, den = tot.s + tot.ey;                   // what the exponentials are relative to in the gradient
        if (kDistill) {
            const DistillTotals totals_row{tot.M, tot.s, tot.ey, zy_row, rest.M, rest.s};
            const DistillOutside outside = distill_outside(s_target[ts], totals_row, r.one_m_py);
            g = -(scale_over_N * dt.tau) * outside.factor;
            den_M = outside.M;
            den = outside.sum;
            if (tid == 0) {
                s_total[ts] = totals_row;
                mbar_arrive(totals(i));
            }
        } else if (!ri.bad_id) {
            if (p.objective == kObjPolicyKl) g = policy_gradient(p, ri.sc, policy_term<true>(p, ri.sc, tot, zy_row), scale_over_N);
            else row_objective<true>(p, ri.sc, tot, zy_row, r.lp, scale_over_N, loss, kl, g);
        }
        if (!kDistill && p.objective != kObjPolicyKl && tid == 0 && crank == 0 && !aborted) {
            if (p.row_loss) p.row_loss[ri.flat] = loss;
            if (p.out_lp_new) p.out_lp_new[ri.flat] = ri.bad_id ? 0.f : r.lp;
        }
        // the policy loss with KL: its terms are formed by one thread, when the block has its gradient
        auto write_terms = [&]() {
            if (kDistill || p.objective != kObjPolicyKl || tid != 0 || crank != 0 || aborted) return;
            float lp = 0.f;
            if (!ri.bad_id) {
                const PolicyTerm q = policy_term<false>(p, ri.sc, tot, zy_row);
                policy_loss_terms(p, ri.sc, q, loss, kl);
                lp = q.lp;
            }
            p.row_loss[ri.flat] = loss;
            p.row_kl[ri.flat] = kl;
            if (p.out_lp_new) p.out_lp_new[ri.flat] = lp;
        };

        // ---- pass 2: gradient = exponential * (-g / sum), written over the logits in the buffer
        uint4* dst = (uint4*)rowbuf + tid;
        if (g == 0.f) {
            for (int j = 0; j < cnt; ++j) dst[(size_t)j * kCons] = make_uint4(0, 0, 0, 0);
        } else {
            // |g| 2^(M - den_M) / den, M this thread's reference.  (Step 4 through lse, whose last place is that of the largest
            // exponent; the others without it, for rows far from 0 and small temperatures.)
            const float mag = kDistill || p.objective != kObjPpo
                                  ? ex2((M - den_M) + (lg2(fabsf(g)) - lg2(den)))
                                  : ex2(M + (lg2(fabsf(g)) - r.lse2));
            const float2 sc2 = splat2(g > 0.f ? -mag : mag);
            const float dy = g * r.one_m_py;
            auto emit = [&](const float2 (&ev)[4], int j) {
                uint32_t o[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float2 d = __fmul2_rn(ev[h], sc2);
                    o[h] = El<kF16>::pack2(d.x, d.y);
                }
                uint4 ov = make_uint4(o[0], o[1], o[2], o[3]);
                if (j == jy) patch_label<kF16>(ov, yj, dy);
                if (j < cnt) dst[(size_t)j * kCons] = ov;
            };
            if (kTmem) tmem_wait_stores();
#pragma unroll
            for (int j = 0; j < kRegVecs; ++j)
                if (j < nj) emit(e[j], j);
            for (int j = 0; kTmem && j < nt; ++j) {
                float2 et[4];
                tmem_load8(tmem_addr + (uint32_t)j * 8u, et);
                tmem_wait_loads();
                emit(et, kRegVecs + j);
            }
        }
        fence_async_smem();                                         // this thread's writes, before the bulk store reads them
        __syncwarp();
        if (lane == 0) mbar_arrive(computed(buf));
        write_terms();
    }
    // The two losses.  Every block leaves its share of the value loss in the workspace; the block that finishes last
    // adds the per-token policy terms (and KL terms, where the objective has them) of the whole batch (all its consumer
    // threads, fixed shares, fixed tree) and the blocks' value-loss shares in block order.
    if (kDistill) asm volatile("bar.sync 2, %0;" ::"n"(kCons + 32) : "memory");   // the patch warp has written the row losses
    if (p.fused) {
        if (tid == 0) {
            p.partials[2 * blockIdx.x] = 0.0;
            p.partials[2 * blockIdx.x + 1] = s_loss[1];
            __threadfence();
            s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1 ? 1 : 0;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kCons) : "memory");
        if (s_last) {
            __threadfence();
            const long long total = (long long)p.B * p.T;
            double acc = 0.0, acc_kl = 0.0;
            if (p.row_loss)
                for (long long q = tid; q < total; q += kCons) acc += (double)__ldcg(p.row_loss + q);
            if (p.row_kl)
                for (long long q = tid; q < total; q += kCons) acc_kl += (double)__ldcg(p.row_kl + q);
            const double pg = consumer_sum_double<NW>(acc, s_dbl, warp, lane);
            const double kl = consumer_sum_double<NW>(acc_kl, s_dbl + 16, warp, lane);
            if (tid == 0) {
                double c = kl;
                for (unsigned k = 0; k < gridDim.x; ++k) c += ((volatile double*)p.partials)[2 * k + 1];
                if (p.out_loss_pg) *p.out_loss_pg = N > 0 ? (float)(pg / (double)D) : 0.f;
                if (p.out_loss_vf) *p.out_loss_vf = N > 0 ? (float)(c / (double)D) : 0.f;
                *p.ticket = 0u;
                if (kCluster == 1) *ca.row_counter = 0u;
            }
        }
    }
    // the tensor-memory columns go back once every consumer is done with them
    if (kTmem) {
        tmem_fence_before_sync();
        asm volatile("bar.sync 1, %0;" ::"n"(kCons) : "memory");
        if (warp == 0) tmem_dealloc(s_tmem_base, ca.tmem_cols);
    }
    if (kCluster > 1) cluster_sync_unaligned();                     // no block leaves while a peer may still write to it
}

}  // namespace rlhf
