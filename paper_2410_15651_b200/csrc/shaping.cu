// Entry points of the operators on shaped logits: argument checks and launches.
#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "host.cuh"
#include "kernels_shaping.cuh"

namespace {

using namespace rlhf;

// Entries of a row and tokens of a history are counted with 32 bits, some turns past their end.
constexpr int kMost = 1 << 30;

// The shaping's arguments into the kernel's form.
int check_shaping(const rlhf_shaping_t* sh, ShapingArgs& out)
{
    if (!sh) return RLHF_ERR_NULL;
    if (sh->prompt_len < 0 || sh->tokens_len < 0 || sh->prompt_len > kMost || sh->tokens_len > kMost) return RLHF_ERR_SHAPE;
    if ((sh->prompt_len > 0 && !sh->prompt) || (sh->tokens_len > 0 && !sh->tokens)) return RLHF_ERR_NULL;
    if (sh->prompt_stride_b < 0 || sh->tokens_stride_b < 0 || sh->bias_stride_b < 0 || sh->mask_stride_b < 0 ||
        sh->mask_stride_t < 0)
        return RLHF_ERR_STRIDE;
    if (!aligned(sh->prompt, 8) || !aligned(sh->tokens, 8) || !aligned(sh->prompt_lengths, 4) || !aligned(sh->start, 4) ||
        !aligned(sh->repetition, 4) || !aligned(sh->frequency, 4) || !aligned(sh->presence, 4) ||
        !aligned(sh->temperature, 4) || !aligned(sh->bias, 4) || !aligned(sh->mask, 4))
        return RLHF_ERR_ALIGN;
    out.tokens = sh->tokens_len > 0 ? sh->tokens : nullptr;
    out.tokens_stride_b = sh->tokens_stride_b;
    out.S = sh->tokens_len;
    out.start = sh->start;
    out.prompt = sh->prompt;
    out.prompt_stride_b = sh->prompt_stride_b;
    out.prompt_lengths = sh->prompt_len > 0 ? sh->prompt_lengths : nullptr;
    out.P = sh->prompt_len;
    out.repetition = sh->repetition;
    out.frequency = sh->frequency;
    out.presence = sh->presence;
    out.temperature = sh->temperature;
    out.bias = sh->bias;
    out.bias_stride_b = sh->bias_stride_b;
    out.mask = sh->mask;
    out.mask_stride_b = sh->mask_stride_b;
    out.mask_stride_t = sh->mask_stride_t;
    return RLHF_OK;
}

// Rows that are read: strides in elements.
int check_read_rows(const void* rows, long long sb, long long st, int T, int V)
{
    if (sb < 0 || st < 0 || (T > 1 && st < V)) return RLHF_ERR_STRIDE;
    return aligned(rows, 2) ? RLHF_OK : RLHF_ERR_ALIGN;
}

// Rows that are written: none overlaps another.
int check_written_rows(const void* rows, size_t size, long long sb, long long st, int B, int T, int V)
{
    if (sb < 0 || st < 0 || (T > 1 && st < V)) return RLHF_ERR_STRIDE;
    if (B > 1 && sb < (T > 1 ? (long long)(T - 1) * st : 0) + V) return RLHF_ERR_STRIDE;
    return aligned(rows, size) ? RLHF_OK : RLHF_ERR_ALIGN;
}

int check_common(int dtype, const int* lengths, int B, int T, int V, const void* ws, size_t ws_bytes)
{
    if (dtype != RLHF_BF16 && dtype != RLHF_F16) return RLHF_ERR_SCALAR;
    if (int e = check_shape(B, T, V)) return e;
    if (V > kMost) return RLHF_ERR_SHAPE;
    if (!aligned(lengths, 4)) return RLHF_ERR_ALIGN;
    return check_workspace(ws, ws_bytes, objective_workspace_bytes(B, T));
}

// Rows whose 16-byte blocks all start at a multiple of 16 bytes from the row (an axis of one position has no stride).
bool rows_aligned(const void* base, size_t size, long long sb, long long st, int B, int T)
{
    const long long per = (long long)(16 / size);
    return aligned(base, 16) && (B == 1 || sb % per == 0) && (T == 1 || st % per == 0);
}

// Blocks (clusters) of the kernel that the device holds at once: they only size the grid.  The answer for the last kernel and
// shape is kept.
template <typename K>
int resident_units(K kernel, int cluster, int threads, size_t smem, const DeviceInfo& dev, int& out)
{
    static std::mutex mu;
    static K of = nullptr;
    static long long key = -1;
    static int value = 0;
    int d = 0;
    RLHF_CUDA(cudaGetDevice(&d));
    const long long k = (((long long)d * 16 + cluster) * 2048 + threads) * 262144 + (long long)smem;
    std::lock_guard<std::mutex> lock(mu);
    if (kernel != of || k != key) {
        int n = 0;
        if (cluster > 1) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            fill_launch_config(cfg, attr, dev.sm_count / cluster * cluster, threads, smem, cluster, nullptr);
            RLHF_CUDA(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
        } else {
            RLHF_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem));
            n *= dev.sm_count;
        }
        value = std::max(n, 1);
        of = kernel;
        key = k;
    }
    out = value;
    return RLHF_OK;
}

template <int kMode, bool kF16, bool kAny>
int launch_shaping_as(ShapeKernelArgs& a, int warps, const DeviceInfo& dev, cudaStream_t s)
{
    void (*kernel)(const ShapeKernelArgs) = nullptr;
    if constexpr (kMode == kShapeLp) kernel = shaping_lp_kernel<kF16, kAny>;
    else kernel = shaping_kernel<kMode, kF16, kAny>;
    const size_t smem = shape_smem(a, warps, kAny).total;
    RLHF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (int e = keep_max_carveout(kernel)) return e;
    // as many blocks as the device holds, each with an equal share of the valid rows (log-probs of few rows: a cluster per row)
    const long long items = (long long)a.B * a.T * (kMode == kShapeLp ? 1 : a.n_slices);
    int units = 0;
    if (int e = resident_units(kernel, a.cluster, warps * 32, smem, dev, units)) return e;
    a.direct = kMode == kShapeLp && (a.T < kShapeShortRows || items <= units);
    const long long grid = (a.direct ? items : std::min<long long>(items, units)) * a.cluster;
    if (grid > 0x7fffffffll) return RLHF_ERR_SHAPE;
    RLHF_CUDA(launch_kernel_cluster(kernel, (int)grid, warps * 32, smem, a.cluster, s, a));
    return launch_check("shaping_kernel");
}

template <int kMode, bool kF16, bool kAny>
int launch_shaping_rows_as(const ShapeKernelArgs& a, cudaStream_t s)
{
    auto kernel = shaping_row_kernel<kMode, kF16, kAny>;
    const size_t smem = shape_row_smem(a, kAny);
    RLHF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (int e = keep_max_carveout(kernel)) return e;
    const long long grid = (long long)a.B * a.T * a.n_slices;
    if (grid > 0x7fffffffll) return RLHF_ERR_SHAPE;
    RLHF_CUDA(launch_kernel(kernel, (int)grid, kRowThreads, smem, s, a));
    return launch_check("shaping_row_kernel");
}

// Words of the bit table and places of the list for a slice of so many entries.
void size_table(ShapeKernelArgs& a, int entries, bool bits)
{
    const long long history = a.uses_history ? (long long)a.sh.P + a.sh.S : 0;
    a.bits_words = a.uses_history || bits ? (entries / 32 + 2 + 3) / 4 * 4 : 0;
    a.list_cap = (int)((std::min<long long>(history, entries) + 1 + 15) / 16 * 16);
}

// Cuts a row into slices and segments, and chooses the kernel.
template <int kMode>
int launch_shaping(ShapeKernelArgs& a, bool f16, bool any, cudaStream_t s)
{
    DeviceInfo dev;
    if (int e = device_info(dev)) return e;
    constexpr bool kLp = kMode == kShapeLp;
    const int vecs = (a.V + (any ? 14 : 7)) / 8;           // most vectors that hold a row's entries
    const long long rows = (long long)a.B * a.T;
    a.wait_limit_ns = kWaitLimitNs;
    a.uses_counts = a.sh.tokens && (a.sh.frequency || a.sh.presence) && kMode != kShapeBwd;
    a.uses_history = (a.sh.repetition && (a.sh.tokens || a.sh.P > 0)) || a.uses_counts;
    a.wide_counts = a.sh.S > 65535;
    a.cluster = 1;

    if constexpr (!kLp) {
        // short sequences, and batches of at most four blocks per SM
        constexpr int kHeld = kRowThreads * kRowVecs;
        const int slices = (vecs + kHeld - 1) / kHeld;
        if (a.T < kShapeShortRows || rows * slices <= 4ll * dev.sm_count) {
            a.n_slices = slices;
            while (rows * a.n_slices < 2ll * dev.sm_count && vecs / a.n_slices > kRowThreads) ++a.n_slices;
            a.segment = (vecs + a.n_slices - 1) / a.n_slices;
            size_table(a, a.segment * 8 + (any ? 16 : 0), false);
            if (any) return f16 ? launch_shaping_rows_as<kMode, true, true>(a, s) : launch_shaping_rows_as<kMode, false, true>(a, s);
            return f16 ? launch_shaping_rows_as<kMode, true, false>(a, s) : launch_shaping_rows_as<kMode, false, false>(a, s);
        }
    }
    // Segments of whole turns of a warp, with two buffers at least.  Log-probs of few rows are cut finer, so that they reach every SM.
    constexpr int kTurn = kLp ? 64 : 32, kWarps = kLp ? kShapeLpWarps : kShapeWarps;
    const size_t room = (size_t)dev.max_smem_optin - 12 * 1024;
    int warps = 0;
    for (a.n_slices = 1;; ++a.n_slices) {
        const int per = (vecs + a.n_slices - 1) / a.n_slices;
        a.segment = ((per + kWarps - 1) / kWarps + kTurn - 1) / kTurn * kTurn;
        warps = std::max(2, (per + a.segment - 1) / a.segment);
        if (a.segment > kShapeSegment) continue;
        if (kLp && a.segment > kTurn && rows * a.n_slices < dev.sm_count && a.n_slices < kShapeMaxCluster) continue;
        size_table(a, a.segment * warps * 8 + (any ? 16 : 0), kLp);
        for (a.n_bufs = kShapeMaxBufs; a.n_bufs > 0 && shape_smem(a, warps, any).total > room; --a.n_bufs) {}
        if (a.n_bufs >= std::min(a.T, 2)) break;
    }
    // log-probs: a row's slices meet in a cluster; what does not fit one is taken in turns
    if (kLp) a.cluster = std::min(a.n_slices, kShapeMaxCluster);
    if (any) return f16 ? launch_shaping_as<kMode, true, true>(a, warps, dev, s) : launch_shaping_as<kMode, false, true>(a, warps, dev, s);
    return f16 ? launch_shaping_as<kMode, true, false>(a, warps, dev, s) : launch_shaping_as<kMode, false, false>(a, warps, dev, s);
}

// Nothing but penalties: outside the history a row is what it was.
bool only_history(const ShapingArgs& sh) { return !sh.bias && !sh.mask && !sh.temperature; }

}  // namespace

extern "C" {

int rlhf_shape_logits(const void* logits, int logits_dtype, long long stride_b, long long stride_t,
                      const rlhf_shaping_t* shaping, const int* lengths, int B, int T, int V,
                      void* out, int out_dtype, long long out_stride_b, long long out_stride_t,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    if (!logits || !lengths || !out) return RLHF_ERR_NULL;
    ShapeKernelArgs a{};
    if (int e = check_shaping(shaping, a.sh)) return e;
    if (int e = check_common(logits_dtype, lengths, B, T, V, workspace, workspace_bytes)) return e;
    if (out_dtype != logits_dtype && out_dtype != RLHF_F32) return RLHF_ERR_SCALAR;
    const size_t size = out_dtype == RLHF_F32 ? 4 : 2;
    if (int e = check_read_rows(logits, stride_b, stride_t, T, V)) return e;
    if (int e = check_written_rows(out, size, out_stride_b, out_stride_t, B, T, V)) return e;
    if (out == logits && (size != 2 || (B > 1 && out_stride_b != stride_b) || (T > 1 && out_stride_t != stride_t)))
        return RLHF_ERR_STRIDE;
    a.src = (const uint16_t*)logits;
    a.src_stride_b = stride_b;
    a.src_stride_t = stride_t;
    a.dst = out;
    a.dst_stride_b = out_stride_b;
    a.dst_stride_t = out_stride_t;
    a.lengths = lengths;
    a.B = B; a.T = T; a.V = V;
    a.status = (unsigned*)workspace;
    a.sparse = out == logits && only_history(a.sh);
    const bool any = !rows_aligned(logits, 2, stride_b, stride_t, B, T) || !rows_aligned(out, size, out_stride_b, out_stride_t, B, T);
    return size == 4 ? launch_shaping<kShape32>(a, logits_dtype == RLHF_F16, any, (cudaStream_t)stream)
                     : launch_shaping<kShape16>(a, logits_dtype == RLHF_F16, any, (cudaStream_t)stream);
}

int rlhf_shape_logits_bwd(const void* dshaped, int logits_dtype, long long ds_stride_b, long long ds_stride_t,
                          const void* logits, long long stride_b, long long stride_t,
                          const rlhf_shaping_t* shaping, const int* lengths, int B, int T, int V,
                          void* out_dlogits, long long dl_stride_b, long long dl_stride_t,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dshaped || !logits || !lengths || !out_dlogits) return RLHF_ERR_NULL;
    ShapeKernelArgs a{};
    if (int e = check_shaping(shaping, a.sh)) return e;
    if (int e = check_common(logits_dtype, lengths, B, T, V, workspace, workspace_bytes)) return e;
    if (int e = check_read_rows(dshaped, ds_stride_b, ds_stride_t, T, V)) return e;
    if (int e = check_read_rows(logits, stride_b, stride_t, T, V)) return e;
    if (int e = check_written_rows(out_dlogits, 2, dl_stride_b, dl_stride_t, B, T, V)) return e;
    if (out_dlogits == logits) return RLHF_ERR_STRIDE;
    if (out_dlogits == dshaped && ((B > 1 && dl_stride_b != ds_stride_b) || (T > 1 && dl_stride_t != ds_stride_t)))
        return RLHF_ERR_STRIDE;
    a.src = (const uint16_t*)dshaped;
    a.src_stride_b = ds_stride_b;
    a.src_stride_t = ds_stride_t;
    a.logits = (const uint16_t*)logits;
    a.logits_stride_b = stride_b;
    a.logits_stride_t = stride_t;
    a.dst = out_dlogits;
    a.dst_stride_b = dl_stride_b;
    a.dst_stride_t = dl_stride_t;
    a.lengths = lengths;
    a.B = B; a.T = T; a.V = V;
    a.status = (unsigned*)workspace;
    a.sparse = out_dlogits == dshaped && !a.sh.mask && !a.sh.temperature;
    const bool any = !rows_aligned(dshaped, 2, ds_stride_b, ds_stride_t, B, T) || !rows_aligned(out_dlogits, 2, dl_stride_b, dl_stride_t, B, T);
    return launch_shaping<kShapeBwd>(a, logits_dtype == RLHF_F16, any, (cudaStream_t)stream);
}

int rlhf_shaped_logprobs(const void* logits, int logits_dtype, long long stride_b, long long stride_t,
                         const long long* ids, long long ids_stride_b, const rlhf_shaping_t* shaping, const int* lengths,
                         int B, int T, int V, float* out_logprobs, float* out_lse, float* out_entropy,
                         void* workspace, size_t workspace_bytes, void* stream)
{
    if (!logits || !ids || !lengths || !out_logprobs || !out_lse) return RLHF_ERR_NULL;
    ShapeKernelArgs a{};
    if (int e = check_shaping(shaping, a.sh)) return e;
    if (int e = check_common(logits_dtype, lengths, B, T, V, workspace, workspace_bytes)) return e;
    if (int e = check_read_rows(logits, stride_b, stride_t, T, V)) return e;
    if (ids_stride_b < 0) return RLHF_ERR_STRIDE;
    if (!aligned(ids, 8) || !aligned(out_logprobs, 4) || !aligned(out_lse, 8) || !aligned(out_entropy, 4)) return RLHF_ERR_ALIGN;
    a.src = (const uint16_t*)logits;
    a.src_stride_b = stride_b;
    a.src_stride_t = stride_t;
    a.lengths = lengths;
    a.B = B; a.T = T; a.V = V;
    a.ids = ids;
    a.ids_stride_b = ids_stride_b;
    a.out_lp = out_logprobs;
    a.out_lse = out_lse;
    a.out_entropy = out_entropy;
    a.status = (unsigned*)workspace;
    const bool any = !rows_aligned(logits, 2, stride_b, stride_t, B, T);
    return launch_shaping<kShapeLp>(a, logits_dtype == RLHF_F16, any, (cudaStream_t)stream);
}

int rlhf_shaped_logprobs_bwd(const void* logits, int logits_dtype, long long stride_b, long long stride_t,
                             const long long* ids, long long ids_stride_b, const rlhf_shaping_t* shaping, const int* lengths,
                             int B, int T, int V, const float* logprobs, const float* lse, const float* entropy,
                             const float* grad_logprobs, const float* grad_entropy,
                             void* out_dlogits, long long dl_stride_b, long long dl_stride_t,
                             void* workspace, size_t workspace_bytes, void* stream)
{
    if (!logits || !ids || !lengths || !logprobs || !lse || !grad_logprobs || !out_dlogits) return RLHF_ERR_NULL;
    if (grad_entropy && !entropy) return RLHF_ERR_NULL;
    ShapeKernelArgs a{};
    if (int e = check_shaping(shaping, a.sh)) return e;
    if (int e = check_common(logits_dtype, lengths, B, T, V, workspace, workspace_bytes)) return e;
    if (int e = check_read_rows(logits, stride_b, stride_t, T, V)) return e;
    if (int e = check_written_rows(out_dlogits, 2, dl_stride_b, dl_stride_t, B, T, V)) return e;
    if (ids_stride_b < 0) return RLHF_ERR_STRIDE;
    if (out_dlogits == logits && ((B > 1 && dl_stride_b != stride_b) || (T > 1 && dl_stride_t != stride_t))) return RLHF_ERR_STRIDE;
    if (!aligned(ids, 8) || !aligned(logprobs, 4) || !aligned(lse, 8) || !aligned(entropy, 4) || !aligned(grad_logprobs, 4) ||
        !aligned(grad_entropy, 4))
        return RLHF_ERR_ALIGN;
    a.src = (const uint16_t*)logits;
    a.src_stride_b = stride_b;
    a.src_stride_t = stride_t;
    a.dst = out_dlogits;
    a.dst_stride_b = dl_stride_b;
    a.dst_stride_t = dl_stride_t;
    a.lengths = lengths;
    a.B = B; a.T = T; a.V = V;
    a.ids = ids;
    a.ids_stride_b = ids_stride_b;
    a.lp = logprobs;
    a.lse = lse;
    a.entropy = entropy;
    a.grad_lp = grad_logprobs;
    a.grad_entropy = grad_entropy;
    a.status = (unsigned*)workspace;
    const bool any = !rows_aligned(logits, 2, stride_b, stride_t, B, T) || !rows_aligned(out_dlogits, 2, dl_stride_b, dl_stride_t, B, T);
    return launch_shaping<kShapeLpBwd>(a, logits_dtype == RLHF_F16, any, (cudaStream_t)stream);
}

}  // extern "C"
