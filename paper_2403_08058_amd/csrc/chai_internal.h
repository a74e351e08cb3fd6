// Internal declarations shared by the translation units of libchai.so (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <stddef.h>
#include <stdint.h>

#include "chai.h"
#include "chai_probe.h"

namespace chai {

constexpr int kHeadDim = 128;       // the only head dimension the kernels are written for
constexpr int kBlock = 256;         // threads per workgroup of the streaming kernels (4 wave64)

// How one decode call is cut into workgroups.  Derived from the sizes alone, so the workspace query and the
// call itself always agree.
struct DecodePlan {
    int cs;          // tokens per workgroup of the score kernel
    int n_cs;        // score chunks per (b, cluster) = ceil(T / cs)
    int n_rec;       // softmax-statistics records per (b, cluster): one per wave of every score workgroup
    int cp;          // tokens per workgroup of the value kernel
    int n_cp;        // value chunks per (b, head) = ceil(T / cp)
    // (off_rows: staging rows of shared values; in other calls the records of 64-token score chunks)
    int ds;          // workgroups per (b, head, chunk) of the value kernel: 1, or 2 with half of the columns each
    size_t off_scores, off_stats, off_partial, off_rows, bytes;   // off_rows: [B,H,128] fp32
};

// row_bytes: bytes of one cached row (rows that are a single cache line are never cut into column parts).  Neither the size of
// the workspace nor what the score phase leaves in it (cs, n_cs, n_rec, off_scores, off_stats) differs between fp32 and bf16
// rows: the two phase calls are planned one by one and each with its own type.
// shared_rows: the H streams' rows are handed out to other heads by a launch of its own (MemberRows below).
DecodePlan make_decode_plan(int B, int H, int k, int T, int row_bytes, bool shared_rows = false);
inline int row_bytes_of(int dtype) { return kHeadDim * (dtype == CHAI_F32 ? 4 : 2); }

// Kernels that use more than 64 KB of dynamic LDS must be told so once on every device they run on.  `done` is the
// caller's per-kernel table (zero-initialised, one flag per device ordinal); a repeated call costs one hipGetDevice.
// The flags are atomics: any thread may call; setting the attribute twice in a race is harmless.
constexpr int kMaxDevices = 64;
typedef std::atomic<bool> DeviceFlags[kMaxDevices];
inline hipError_t allow_dynamic_lds(const void *kernel, size_t bytes, DeviceFlags &done)
{
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 0 && dev < kMaxDevices && done[dev].load(std::memory_order_acquire)) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess && dev >= 0 && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
    return e;
}

// Optional events the runtime stamps with the begin and the end of a kernel (NULL = not wanted).
struct KernelEvents {
    hipEvent_t start = nullptr;
    hipEvent_t stop = nullptr;
};

// Kernel launch that reports the status of THIS launch: the return value of the runtime's launch call, not the
// thread's sticky "last error" (which may hold, and would clear, an unrelated earlier error of the caller).
// Arguments are converted to the kernel's own parameter types; the events may be NULL.
template <typename T>
struct same_type {
    typedef T type;
};
template <typename... KArgs>
inline hipError_t launch_kernel(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds_bytes, hipStream_t stream,
                                const KernelEvents &ev, typename same_type<KArgs>::type... args)
{
    void *argv[] = {const_cast<void *>(static_cast<const void *>(&args))...};
    return hipExtLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, argv, lds_bytes, stream, ev.start,
                              ev.stop, 0);
}

// Enqueue the two kernels of one decode call.  identity = true: every head is its own cluster and the maps
// are not read (dense attention).  k_new / v_new [B,H,d] (clustered calls only): position T-1 is the token being
// decoded, its rows are taken from there and written to the caches by the same kernels.  Each returns a
// hipError_t as int.
int launch_scores(const void *q, const void *kc, const int32_t *rep, int B, int H, int k, int T, int Tc_cap,
                  int dtype, float scale, void *workspace, const DecodePlan &plan, bool identity,
                  const KernelEvents &ev, hipStream_t stream, const void *k_new = nullptr);
// Both phases of one call, in two launches or, for dense and for small calls, in one (plus the sum of partial rows); no copy of the
// probabilities.
int launch_decode(const void *q, const void *kc, const void *v, const int32_t *h2c, const int32_t *rep, int B, int H, int k, int T,
                  int Tc_cap, int T_cap, int dtype, float scale, float *out, void *workspace, const DecodePlan &plan, bool identity,
                  hipStream_t stream, const void *k_new = nullptr, const void *v_new = nullptr);
// members: when set, the H streams of `v` are compact (one per cluster) and the finished row of stream j goes
// to out_members[b][h] of every head h (of n_heads) with head_to_cluster[b][h] == j; `out` is then staging.
struct MemberRows {
    const int32_t *head_to_cluster = nullptr;
    int n_heads = 0;
    float *out_members = nullptr;
};
int launch_values(const void *v, const int32_t *h2c, const int32_t *rep, int B, int H, int k, int T, int T_cap,
                  int dtype, float *out, float *probs_out, void *workspace, const DecodePlan &plan, bool identity,
                  const KernelEvents &ev, hipStream_t stream, const MemberRows *members = nullptr,
                  const void *v_new = nullptr);

// The same two kernels over caches of 8-bit E4M3 codes with one fp32 scale per row; q stays fp32 or bf16 (q_dtype).
// The plan must have been made for rows of kHeadDim bytes.
int launch_scores_q8(const void *q, int q_dtype, const void *k8, const float *kscale, const int32_t *rep, int B, int H,
                     int k, int T, int Tc_cap, float scale, void *workspace, const DecodePlan &plan,
                     const KernelEvents &ev, hipStream_t stream);
int launch_values_q8(const void *v8, const float *vscale, const int32_t *h2c, const int32_t *rep, int B, int H, int k,
                     int T, int T_cap, float *out, float *probs_out, void *workspace, const DecodePlan &plan,
                     const KernelEvents &ev, hipStream_t stream);
// rows of 128 elements (fp32 / bf16) -> E4M3 codes + one fp32 scale per row
int launch_quantize_rows(const void *x, int dtype, long long n_rows, uint8_t *codes, float *scales, hipStream_t stream);
int launch_append_kv_q8(const void *k_new, const void *v_new, const int32_t *rep, uint8_t *k8, float *kscale, uint8_t *v8,
                        float *vscale, int B, int H, int k, int pos, int Tc_cap, int T_cap, int dtype,
                        hipStream_t stream);

int launch_score_features(const void *q5, const void *k5, int B, int H, int n_tok, int dtype, int64_t qs,
                          int64_t ks, float scale, float *feat, hipStream_t stream);

int launch_assign_clusters(const float *feat, int B, int H, int F, int k, const int32_t *init_heads, int max_iter,
                           int32_t *h2c, int32_t *rep, int32_t *ncl, int32_t *iters, hipStream_t stream);
bool assign_clusters_supported(int H, int F, int k);

// sse and rep_out (nearest-to-mean member of every cluster) are optional outputs of the same kernel
int launch_cluster_error(const float *feat, const int32_t *h2c, int B, int H, int F, int k, double *sse,
                         int32_t *rep_out, hipStream_t stream);
size_t cluster_error_lds_bytes(int H, int F, int k);

// Clustered attention over a block of prompt positions (bf16 only).  identity = dense attention.  The events
// cover the main kernel, not the V^T pre-pass or the work list.
int launch_prefill(const void *q, const void *kc, const void *v, const int32_t *h2c, const int32_t *rep, int B,
                   int H, int k, int Tq, int q_start, int Tc_cap, int T_cap, float scale, float *out,
                   void *workspace, bool identity, const KernelEvents &ev, hipStream_t stream);
size_t prefill_workspace_bytes(int B, int H, int k, int n_keys);

// Query and key projections of the representatives (bf16, d = 128, D a multiple of 64); the events cover the kernel.
int launch_project_qk(const void *x, const void *w_q, const void *w_k, const int32_t *rep, int B, int H, int k, int Tn,
                      int D, void *q_out, void *k_compact, int pos0, int Tc_cap, const KernelEvents &ev,
                      hipStream_t stream);

// The same with a low-rank adapter of every row's own: first t = s_a x A_a^T of all tokens, then the projections, which add t B_a^T.
struct AdapterUse {
    const char *t = nullptr;             // [B,Tn][2 (queries, keys)][chunks][upper | middle | lower 8 bits of 16 ranks] bf16
    const char *b_q = nullptr, *b_k = nullptr;           // [n,H*128,R] bf16, or NULL: none of that part
    const int32_t *ids = nullptr;        // [B]
    int n = 0, R = 0;
    __host__ __device__ int chunks() const { return (R + 15) / 16; }
};
constexpr int kMaxAdapterRank = 128;
constexpr int kAdapterChunkBytes = 3 * 16 * 2;           // of t: sixteen ranks, three bf16 each
size_t adapter_workspace_bytes(int B, int Tn, int R);
int launch_adapter_down(const void *x, const int32_t *ids, const void *a_q, const void *a_k, const float *scales, int n, int R, int B, int Tn,
                        int D, void *t, hipStream_t stream);
int launch_project_qk_adapted(const void *x, const void *w_q, const void *w_k, const int32_t *rep, int B, int H, int k, int Tn, int D,
                              void *q_out, void *k_compact, int pos0, int Tc_cap, const AdapterUse &use, hipStream_t stream);

// Caches in pages.  rows of either kind: [n_pages, streams, page, 128], streams = k for keys and H for values.
struct PagedShape {
    const int32_t *table = nullptr;      // [B, max_blocks]: page of positions [i * page, (i + 1) * page) of a row
    const int32_t *lens = nullptr;       // [B]
    int B = 0, H = 0, k = 0, T_max = 0, n_pages = 0, page = 0, max_blocks = 0;
    int div_shift = 0;                   // n / page without a division (set_page_division)
    unsigned int div_mul = 0;
};
struct PagedPages {
    const char *k = nullptr, *v = nullptr;
    const float *k_scales = nullptr, *v_scales = nullptr;
};
// Regions of the workspace, upper bounds over the types.
struct PagedPlan {
    size_t off_recs, off_partial, off_whole, off_scores, bytes;
};
constexpr int kMaxPagedBatch = 4096;     // rows: two levels of 64 lanes add up their lengths
constexpr int kMaxPagedTokens = 1 << 24;
PagedPlan make_paged_plan(int B, int H, int k, int T_max);
void set_page_division(PagedShape *sh);
// h2c = rep = NULL: every head its own cluster (k = H).  k_new / v_new [B,H,d] (or NULL): the last position of every row is the token
// being decoded, its rows are taken from there and written to the pages by the same kernels.
int launch_paged_attention(const PagedShape &sh, const PagedPages &pg, const void *q, const void *k_new, const void *v_new, int dtype,
                           int cache_dtype, const int32_t *h2c, const int32_t *rep, float scale, float *out, void *workspace,
                           const PagedPlan &plan, hipStream_t stream);
int launch_paged_append(const PagedShape &sh, const PagedPages &pg, const void *k_new, const void *v_new, int64_t k_stride,
                        int64_t v_stride, const int32_t *rep, const int32_t *start, const int32_t *count, int Tn, int dtype,
                        int cache_dtype, hipStream_t stream);
int launch_paged_gather(const PagedShape &sh, const PagedPages &pg, const int32_t *start, const int32_t *count, void *k_out, void *v_out,
                        int Tn, int dtype, int cache_dtype, hipStream_t stream);

// Places of new tokens (chai_paged_place_tokens): all pointers on the device.
struct PlaceShape {
    int B = 0, N = 0, n_pages = 0, page = 0, max_blocks = 0;
    int div_shift = 0;                   // n / page without a division
    unsigned int div_mul = 0;
};
struct PlaceIn {
    const int32_t *counts = nullptr, *lens = nullptr, *free_pages = nullptr, *n_free = nullptr;
};
struct PlaceOut {
    int32_t *table = nullptr, *new_lens = nullptr, *n_left = nullptr, *granted = nullptr, *offsets = nullptr, *token_rows = nullptr,
            *positions = nullptr, *slots = nullptr;
};
size_t place_workspace_bytes(int B);
int launch_place_tokens(const PlaceShape &sh, const PlaceIn &in, const PlaceOut &out, void *workspace, hipStream_t stream);
int launch_release_pages(const PlaceShape &sh, const int32_t *keep, const int32_t *lens, int32_t *table, int32_t *free_pages,
                         const int32_t *n_free, int32_t *new_lens, int32_t *n_left, hipStream_t stream);

// Rows turned by their positions: blocks of tokens of a contiguous cache, or tokens one behind the other on their way into pages.
struct TurnShape {
    const int32_t *rep = nullptr;        // [B,k], or NULL: every head (k = H)
    const int32_t *positions = nullptr;  // of every token, or NULL (blocks): pos0 + its number
    const double *freq = nullptr;        // [rot / 2] radians per position
    int B = 0, H = 0, k = 0, rot = 0;
    double gain = 1.0;
    int Tn = 0, pos0 = 0, Tc_cap = 0;    // blocks: n = b * Tn + i
    const int32_t *rows = nullptr, *slots = nullptr;     // packed: of every token
    int N = 0, by_slot = 0, n_pages = 0, page = 0, div_shift = 0;
    unsigned int div_mul = 0;
};
struct TurnRows {
    const char *q = nullptr, *k = nullptr, *v = nullptr;
    long long q_stride = 0, k_stride = 0, v_stride = 0;  // elements from head to head (blocks) or token to token (packed)
    long long out_stride = 0, q_head = 0, k_head = 0, v_head = 0, out_head = 0;          // packed: of q_out; from head to head
    char *q_out = nullptr, *k_out = nullptr, *v_out = nullptr;       // (k_out, v_out: caches or pages)
    float *k_scales = nullptr, *v_scales = nullptr;
};
int launch_rotate(const TurnShape &sh, const TurnRows &rows, int layout, int dtype, hipStream_t stream);
int launch_append_packed(const TurnShape &sh, const TurnRows &rows, int layout, int dtype, int cache_dtype, hipStream_t stream);

// 32 x 32 x 16 products alone: `rounds` rounds of 8 of them per wave on operands taken from buf; flops of one launch
int launch_mfma_probe(const void *buf, size_t bytes, int rounds, float *sink, const KernelEvents &ev, hipStream_t stream);
double mfma_probe_flops(int rounds);

// bare streaming read of `bytes` (a multiple of 16) bytes; the events cover the kernel
int launch_stream_read(const void *buf, size_t bytes, float *sink, const KernelEvents &ev, hipStream_t stream);

int launch_compact_kcache(const void *k_full, const int32_t *rep, void *k_compact, int B, int H, int k, int T,
                          int T_cap, int Tc_cap, int dtype, hipStream_t stream);

// Both caches compact (the variant that prunes values too): rows of the representatives only.
int launch_append_kv_shared(const void *k_new, const void *v_new, const int32_t *rep, void *k_compact, void *v_compact,
                            int B, int H, int k, int pos, int Tc_cap, int Tv_cap, int dtype, hipStream_t stream);

int launch_append_kv(const void *k_new, const void *v_new, const int32_t *rep, void *k_compact, void *v_cache, int B,
                     int H, int k, int pos, int Tc_cap, int T_cap, int dtype, hipStream_t stream);

}  // namespace chai
