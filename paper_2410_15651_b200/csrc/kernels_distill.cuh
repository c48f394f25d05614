// Distillation from a teacher's entries for rows outside the range of loss_creg_kernel<..., kDistill> (kernels_creg.cuh):
// rows shorter than 16 KB or longer than a cluster of four blocks holds, rows off 16-byte boundaries that one block does not hold
// (more than 53241 entries), and gradient rows laid out off their logits rows' 16-byte boundaries.
//
// A rare case is served plainly: the kernel is bound by its own instructions, not by DRAM.  4096 rows, bf16, K = 64: V = 1000 81 us,
// 8176 164 us (floor 20), 53249 534 us (133), 100277 964 us (250; V = 100280 on the fast kernel 277), 151643 1427 us; V = 50272
// with gradients at another offset 607 us (146 at the same).
//
// One block per row, dealt statically; the row is read twice, the second time from L2.  The teacher's entries go into a
// small hash table in shared memory (entry -> position in the list); a bitmap over the row's 16-byte vectors (mod 4096)
// says for most vectors that none of their entries is in it.  As in the other kernel the sum over the entries that are
// not the teacher's is formed without them, and entries named twice add their weights in the order of the list.
#pragma once
#include "kernels_creg.cuh"
#include "kernels_objective.cuh"
#include "kernels_topk.cuh"

namespace rlhf {

constexpr int kDistillThreads = 256;
constexpr int kDistillSlots = 512;          // hash table: at most half full
constexpr int kDistillMapWords = 128;       // bitmap of 4096 bits

struct DistillRowArgs {
    RowArgs row;                // row_loss, out_lp_new = per-row loss (optional)
    DistillArgs distill;
    int same_offsets;           // gradient rows lie as far off 16-byte boundaries as their logits rows
};

struct DistillTable {
    int key[kDistillSlots];     // entry, or -1
    int k[kDistillSlots];       // its first position in the list
    uint32_t map[kDistillMapWords];
};

__device__ __forceinline__ uint32_t distill_hash(int id) { return ((uint32_t)id * 2654435769u) >> 23; }
static_assert(kDistillSlots == 1 << 9, "distill_hash keeps 9 bits");

// Position in the list of entry `id`, or -1.
__device__ __forceinline__ int distill_find(const DistillTable& tab, int id)
{
    uint32_t h = distill_hash(id);
    for (int n = 0; n < kDistillSlots; ++n, h = (h + 1) & (kDistillSlots - 1)) {
        const int key = tab.key[h];
        if (key == id) return tab.k[h];
        if (key < 0) return -1;
    }
    return -1;
}

template <bool kF16>
__global__ void __launch_bounds__(kDistillThreads) distill_row_kernel(DistillRowArgs da)
{
    __shared__ DistillTable s_tab;
    __shared__ int s_id[kDistillMax];
    __shared__ float s_p[kDistillMax], s_grad[kDistillMax];
    __shared__ double s_red[kDistillThreads / 32];
    __shared__ float s_f[kDistillThreads / 32];
    __shared__ Acc s_acc[32];
    __shared__ long long s_cnt[33];
    __shared__ TargetInfo s_ti;
    __shared__ int s_twice;
    __shared__ DistillTotals s_tot;
    const RowArgs& p = da.row;
    const DistillArgs& dt = da.distill;
    const int tid = threadIdx.x;
    pdl_wait_prior_grid();
    pdl_release_next_grid();
    const long long N = block_count_valid(p.lengths, p.B, p.T, s_cnt, blockIdx.x == 0 ? p.status : nullptr);
    const float row_scale = N > 0 ? p.grad_scale * dt.tau / (float)N : 0.f;

    // block-wide maximum or sum of one float, for every thread
    auto block_max = [&](float v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        __syncthreads();
        if ((tid & 31) == 0) s_f[tid >> 5] = v;
        __syncthreads();
        for (int w = 0; w < kDistillThreads / 32; ++w) v = fmaxf(v, s_f[w]);
        return v;
    };
    auto block_add = [&](double v) {
        const double t = block_sum_double<kDistillThreads>(v, s_red);
        __syncthreads();
        if (tid == 0) s_red[0] = t;
        __syncthreads();
        return s_red[0];
    };

    Cursor cur{0, 0};
    for (long long row = blockIdx.x; row < N; row += gridDim.x) {
        int b, t;
        if (!cursor_seek_valid(cur, row, p.lengths, p.B, p.T, b, t)) break;
        const long long flat = (long long)b * p.T + t;
        const uint16_t* z16 = p.logits + (long long)b * p.stride_b + (long long)t * p.stride_t;
        uint16_t* d16 = p.dlogits + (long long)b * p.dl_stride_b + (long long)t * p.dl_stride_t;
        const long long entries = (long long)b * dt.stride_b + (long long)t * dt.stride_t;

        // ---- the teacher's entries: thread k has entry k
        __syncthreads();
        for (int i = tid; i < kDistillSlots; i += kDistillThreads) { s_tab.key[i] = -1; s_tab.k[i] = kDistillMax; }
        for (int i = tid; i < kDistillMapWords; i += kDistillThreads) s_tab.map[i] = 0;
        if (tid == 0) s_twice = 0;
        int id = -1;
        float lt = __uint_as_float(0xff800000u);
        if (tid < dt.K) {
            id = __ldg(dt.ids + entries + tid);
            if (id < -1 || id >= p.V) atomicOr(p.status, kErrIdRange);
            if (id < 0 || id >= p.V) id = -1;
            else lt = __ldg(dt.logprobs + entries + tid);
        }
        float pk;
        double P;
        if (dt.mode == kDistillNormalised) {
            const float m = block_max(fmaxf(lt, kFloorM));
            pk = expf(lt - m);
            P = block_add((double)pk);
            const float inv = P > 0.0 ? (float)(1.0 / P) : (P == P ? 0.f : (float)P);
            pk *= inv;
            lt -= m + (float)log(P);
            P = P > 0.0 ? 1.0 : (P == P ? 0.0 : P);
        } else {
            const double e = exp((double)lt);
            pk = dt.mode == kDistillTail ? (float)e : expf(lt);
            P = block_add(dt.mode == kDistillTail ? e : (double)pk);
        }
        const double H = block_add(pk == 0.f ? 0.0 : (double)pk * (double)lt);
        if (tid < dt.K) { s_id[tid] = id; s_p[tid] = pk; }
        // (the sums above have a barrier behind the table's clearing)
        uint32_t slot = 0;
        if (id >= 0) {
            slot = distill_hash(id);
            for (int n = 0; n < kDistillSlots; ++n, slot = (slot + 1) & (kDistillSlots - 1)) {
                const int was = atomicCAS(&s_tab.key[slot], -1, id);
                if (was == -1 || was == id) break;
            }
            atomicMin(&s_tab.k[slot], tid);
        }
        const RowSpan r = row_span(z16, p.V);
        if (id >= 0) {
            const uint32_t v = ((r.eoff + (uint32_t)id) >> 3) & (kDistillMapWords * 32 - 1);
            atomicOr(&s_tab.map[v >> 5], 1u << (v & 31));
        }
        __syncthreads();
        const bool first = id >= 0 && s_tab.k[slot] == tid;
        if (id >= 0 && !first) s_twice = 1;
        __syncthreads();
        if (s_twice && first)
            for (int o = tid + 1; o < dt.K; ++o)
                if (s_id[o] == id) pk += s_p[o];
        float z = 0.f, x = kFloorM;
        if (first) { z = El<kF16>::widen(z16[id]); x = fmaxf(z * dt.scale, kFloorM); }
        const float Mt = block_max(x);
        const float xr = first ? fmaf(z, dt.scale, -Mt) : 0.f;

        // ---- pass 1: sum over the entries that are not the teacher's, against the largest of the vector maxima
        float M = kFloorM, s = 0.f;
        auto may_hold = [&](uint32_t v) { return (s_tab.map[(v >> 5) & (kDistillMapWords - 1)] >> (v & 31)) & 1u; };
        for (uint32_t v = tid; v < r.nvec; v += kDistillThreads) {
            uint4 q = *(r.vecs + v);
            if (v == 0 || v == r.nvec - 1)
                q = mask_vec_outside<kF16>(q, v == 0 ? (int)r.eoff : 0, v == r.nvec - 1 ? (int)r.tail : 8);
            if (may_hold(v))
                for (int i = 0; i < 8; ++i) {
                    const int e = (int)(v * 8u + (uint32_t)i) - (int)r.eoff;
                    if (e >= 0 && e < p.V && distill_find(s_tab, e) >= 0) q = mask_vec_entry<kF16>(q, i);
                }
            float zz[8], vs = 0.f;
            unpack8<kF16>(q, zz);
            float m = fmaxf(fmaxf(fmaxf(zz[0], zz[1]), fmaxf(zz[2], zz[3])), fmaxf(fmaxf(zz[4], zz[5]), fmaxf(zz[6], zz[7])));
            m = fmaxf(m * dt.scale, M);
#pragma unroll
            for (int i = 0; i < 8; ++i) vs += ex2(fmaf(zz[i], dt.scale, -m));
            s = fmaf(s, ex2(M - m), vs);
            M = m;
        }
        const double ey = block_add(first ? (double)ex2(xr) : 0.0);
        const double zy = block_add(first && !(pk == 0.f) ? (double)pk * (double)xr : 0.0);
        Acc a = block_merge(Acc{M, s, 0.f}, s_acc);
        if (tid == 0) {
            TargetInfo ti{};
            ti.H = H;
            ti.P = (float)P;
            ti.p0 = dt.mode == kDistillTail ? (float)(1.0 - P > 0.0 ? 1.0 - P : 0.0) : 0.f;
            ti.W = dt.mode == kDistillTail ? (float)(P > 1.0 ? P : 1.0) : (float)P;
            if (!(P == P)) ti.W = ti.P;
            const float Mx = fmaxf(a.M, Mt);
            const DistillTotals tot{Mx, a.s * ex2(a.M - Mx), (float)ey * ex2(Mt - Mx), fmaf((float)P, Mt - Mx, (float)zy), a.M, a.s};
            s_ti = ti;
            s_tot = tot;
            const float L = (float)((double)dt.tau * (double)dt.tau * distill_loss(ti, tot));
            p.row_loss[flat] = L;
            if (p.out_lp_new) p.out_lp_new[flat] = L;
        }
        __syncthreads();
        const DistillTotals tot = s_tot;
        const TargetInfo ti = s_ti;
        if (first)
            s_grad[tid] = row_scale * fmaf(distill_weight(ti, tot.so), ex2(fmaf(z, dt.scale, -tot.M) - log2f(tot.s + tot.ey)), -pk);
        __syncthreads();

        // ---- pass 2: the gradient
        const DistillOutside outside = distill_outside(ti, tot, tot.s / (tot.s + tot.ey));
        const float f = row_scale * outside.factor, l2 = log2f(outside.sum);
        for (uint32_t v = tid; v < r.nvec; v += kDistillThreads) {
            const uint4 q = *(r.vecs + v);
            float zz[8];
            unpack8<kF16>(q, zz);
            const bool named = may_hold(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                zz[i] = f == 0.f ? 0.f : f * ex2(fmaf(zz[i], dt.scale, -outside.M) - l2);
                const int e = (int)(v * 8u + (uint32_t)i) - (int)r.eoff;
                if (named && e >= 0 && e < p.V) {
                    const int k = distill_find(s_tab, e);
                    if (k >= 0) zz[i] = s_grad[k];
                }
            }
            const uint4 o = make_uint4(El<kF16>::pack2(zz[0], zz[1]), El<kF16>::pack2(zz[2], zz[3]),
                                       El<kF16>::pack2(zz[4], zz[5]), El<kF16>::pack2(zz[6], zz[7]));
            const int e0 = (int)(v * 8u) - (int)r.eoff;
            if (da.same_offsets && e0 >= 0 && e0 + 8 <= p.V) {
                *(uint4*)(d16 + e0) = o;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (e0 + i >= 0 && e0 + i < p.V) d16[e0 + i] = (uint16_t)vec_entry(o, i);
            }
        }
    }
    // zero rows for padded tokens
    const long long n_pad = (long long)p.B * p.T - N;
    Cursor pc{0, 0};
    for (long long k = blockIdx.x; k < n_pad; k += gridDim.x) {
        int b, t;
        if (!cursor_seek_padded(pc, k, p.lengths, p.B, p.T, b, t)) break;
        uint16_t* d16 = p.dlogits + (long long)b * p.dl_stride_b + (long long)t * p.dl_stride_t;
        const RowSpan r = row_span(d16, p.V);
        for (uint32_t v = tid; v < r.nvec; v += kDistillThreads) {
            const int e0 = (int)(v * 8u) - (int)r.eoff;
            if (e0 >= 0 && e0 + 8 <= p.V) *(uint4*)(d16 + e0) = make_uint4(0, 0, 0, 0);
            else
                for (int i = 0; i < 8; ++i)
                    if (e0 + i >= 0 && e0 + i < p.V) d16[e0 + i] = 0;
        }
    }
}

}  // namespace rlhf
