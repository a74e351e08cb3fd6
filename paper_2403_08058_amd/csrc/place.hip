// Places of new tokens: which rows of a batch get their new tokens, which pages of a list of free ones they take for them, and where
// every token of the batch, one row's behind the other's, then stands.  All on the device: lengths, tables and the list never come to
// the host, so that a recorded step can be replayed while rows grow.
//
//   row b:    have = ceil(len / page) pages, need = ceil((len + count) / page) - have more, granted iff its tokens end within the block
//             of N tokens and within its table, and need = 0 or need[0] + .. + need[b] <= n_free (over the rows that end within both)
//   pages:    the list is a stack; the rows take from its top, in row order
//   token i:  position len + i in page position / page of its row, slot = page number * page + position % page
//
// Two sums over the rows (tokens and pages), both capped, so that no number of tokens overflows them: min(a + b, cap) is associative.
//
// What bounds it: look-ups that depend on one another (lengths, two sums over the workgroup, the row of a token, its page) and the launch.
#include "chai_internal.h"

#include <hip/hip_ext.h>

namespace chai {

namespace {

constexpr int kPlaceBlock = 256;
constexpr int kPlaceWaves = kPlaceBlock / 64;
constexpr int kPlaceOneTokens = 2048;        // that one workgroup takes at most
constexpr int kPlaceMost = 1024;             // workgroups of a launch that all look at the rows

__device__ __forceinline__ unsigned int capped(unsigned int a, unsigned int b, unsigned int cap) { return min(a + b, cap); }

// position / page, as the attention kernels find it
__device__ __forceinline__ int block_at(const PlaceShape &sh, unsigned int pos) { return (int)((__umulhi(pos, sh.div_mul) + pos) >> sh.div_shift); }
__device__ __forceinline__ int blocks_of(const PlaceShape &sh, unsigned int n) { return n == 0u ? 0 : block_at(sh, n - 1u) + 1; }

// What the tokens of a row have to know of it.
struct PlacedRow {
    int first;        // number of its first token in the block
    int len;          // positions before the call
    int have;         // its pages before the call, or -1: it got none of what it asked for
    int top;          // its i-th new page is free_pages[top - 1 - i]
};

// inclusive sum over the workgroup, capped; `sums` [kPlaceWaves] is free again after the call's barrier and one more
__device__ __forceinline__ unsigned int block_scan(unsigned int x, unsigned int cap, unsigned int *sums)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned int other = (unsigned int)__shfl_up((int)x, o);
        if (lane >= o) x = capped(x, other, cap);
    }
    if (lane == 63) sums[w] = x;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kPlaceWaves; ++v)
        if (v < w) x = capped(x, sums[v], cap);
    return x;
}

// Which rows get their tokens; a workgroup, SPAN rows a thread.  rows: [B] in LDS or in the workspace; total (in LDS or NULL): tokens of all;
// `write`: the rows' outputs, by one of the workgroups that find the same.  Everything that may be written in place (new_lens over
// seq_lens, n_left over n_free) has been read by every thread before the first barrier.
template <int SPAN>
__device__ __forceinline__ void place_rows(const PlaceShape &sh, const PlaceIn &in, const PlaceOut &out, PlacedRow *rows, int *total, bool write)
{
    __shared__ unsigned int sums[2][kPlaceWaves], taken;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, b0 = tid * SPAN;
    const unsigned int most_tokens = (unsigned int)sh.N + 1u, most_pages = (unsigned int)sh.n_pages + 1u;
    int given[SPAN], len[SPAN];
#pragma unroll
    for (int i = 0; i < SPAN; ++i) {                     // (rows past the end ask for nothing)
        given[i] = b0 + i < sh.B ? in.counts[b0 + i] : 0;
        len[i] = b0 + i < sh.B ? max(in.lens[b0 + i], 0) : 0;
    }
    const unsigned int n_free = (unsigned int)min(max(in.n_free[0], 0), sh.n_pages);
    const long long reach = min((long long)sh.max_blocks * sh.page, 0x7fffffffll);
    if (tid == 0) taken = 0u;

    // what came before a thread's rows: with a cap it cannot be had from the sum up to them by subtraction
    auto before = [&](unsigned int upto, const unsigned int *of_waves, unsigned int cap) {
        unsigned int x = (unsigned int)__shfl_up((int)upto, 1);
        if (lane == 0) {
            x = 0u;
            for (int v = 0; v < w; ++v) x = capped(x, of_waves[v], cap);
        }
        return x;
    };
    unsigned int count[SPAN], tokens = 0u;
#pragma unroll
    for (int i = 0; i < SPAN; ++i) {
        count[i] = min((unsigned int)max(given[i], 0), most_tokens);
        tokens = capped(tokens, count[i], most_tokens);
    }
    const unsigned int tokens_upto = block_scan(tokens, most_tokens, sums[0]);
    unsigned int first[SPAN], need[SPAN], end = before(tokens_upto, sums[0], most_tokens), pages = 0u;
    bool fits[SPAN];
#pragma unroll
    for (int i = 0; i < SPAN; ++i) {
        first[i] = end;
        end = capped(end, count[i], most_tokens);
        fits[i] = end <= (unsigned int)sh.N && (long long)len[i] + count[i] <= reach;
        need[i] = fits[i] ? (unsigned int)(blocks_of(sh, (unsigned int)len[i] + count[i]) - blocks_of(sh, (unsigned int)len[i])) : 0u;
        pages = capped(pages, need[i], most_pages);
    }
    const unsigned int pages_upto = block_scan(pages, most_pages, sums[1]);
    unsigned int pages_end = before(pages_upto, sums[1], most_pages), last = 0u;
#pragma unroll
    for (int i = 0; i < SPAN; ++i) {
        const int b = b0 + i;
        const unsigned int pages_before = pages_end;
        pages_end = capped(pages_end, need[i], most_pages);
        const bool granted = fits[i] && (need[i] == 0u || pages_end <= n_free);
        if (granted && need[i] != 0u) last = pages_end;
        if (b >= sh.B) continue;
        const int at = (int)min(first[i], (unsigned int)sh.N);
        rows[b] = PlacedRow{at, len[i], granted ? blocks_of(sh, (unsigned int)len[i]) : -1, granted ? (int)(n_free - min(pages_before, n_free)) : 0};
        if (write) {
            out.offsets[b] = at;
            out.granted[b] = granted ? 1 : 0;
            out.new_lens[b] = granted ? len[i] + (int)count[i] : len[i];
        }
    }
    if (last != 0u) atomicMax(&taken, last);
    if (tid == kPlaceBlock - 1) {
        if (write) out.offsets[sh.B] = (int)min(tokens_upto, (unsigned int)sh.N);
        if (total != nullptr) *total = (int)min(tokens_upto, (unsigned int)sh.N);
    }
    __syncthreads();
    if (tid == 0 && write) out.n_left[0] = (int)(n_free - taken);
}

// Token n: its row (the last one that begins at or before it: rows without tokens begin where the next one does), position and slot;
// the first token of a page that its row took enters it in the table.
__device__ __forceinline__ void place_token(const PlaceShape &sh, const PlaceIn &in, const PlaceOut &out, const PlacedRow *rows, int n, int total)
{
    int b = -1, pos = 0, slot = -1;
    if (n < total) {
        int lo = 0, hi = sh.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (rows[mid].first <= n) lo = mid;
            else hi = mid - 1;
        }
        b = lo;
        const PlacedRow r = rows[b];
        const unsigned int at = (unsigned int)r.len + (unsigned int)(n - r.first);
        pos = (int)at;
        if (r.have >= 0) {
            const int block = block_at(sh, at), place = (int)at - block * sh.page;
            int32_t *entry = out.table + (size_t)b * sh.max_blocks + block;
            int p;
            if (block >= r.have) {
                p = in.free_pages[r.top - 1 - (block - r.have)];
                if (place == 0) *entry = p;
            } else {
                p = *entry;
            }
            if ((unsigned int)p < (unsigned int)sh.n_pages) slot = p * sh.page + place;
        }
    }
    out.token_rows[n] = b;
    out.positions[n] = pos;
    out.slots[n] = slot;
}

// One launch for everything.  Where there are many tokens several workgroups take them, each of which finds out about the rows for itself
// (nothing that they read may be written in place then: only the first writes what is known of rows, but it does not wait for the others).
template <int SPAN>
__global__ __launch_bounds__(kPlaceBlock) void place_all_kernel(PlaceShape sh, PlaceIn in, PlaceOut out)
{
    __shared__ PlacedRow rows[SPAN * kPlaceBlock];
    __shared__ int total;
    place_rows<SPAN>(sh, in, out, rows, &total, blockIdx.x == 0);
    for (int n = blockIdx.x * kPlaceBlock + threadIdx.x; n < sh.N; n += gridDim.x * kPlaceBlock) place_token(sh, in, out, rows, n, total);
}

template <int SPAN>
__global__ __launch_bounds__(kPlaceBlock) void place_rows_kernel(PlaceShape sh, PlaceIn in, PlaceOut out, PlacedRow *rows)
{
    place_rows<SPAN>(sh, in, out, rows, nullptr, true);
}

__global__ __launch_bounds__(kPlaceBlock) void place_tokens_kernel(PlaceShape sh, PlaceIn in, PlaceOut out, const PlacedRow *rows)
{
    const int n = blockIdx.x * kPlaceBlock + threadIdx.x;
    if (n < sh.N) place_token(sh, in, out, rows, n, out.offsets[sh.B]);
}

// ---------------------------------------------------------------------------------------------------------
// Pages of rows that end, or lose their last positions, go back on the list: those behind the kept positions that are pages, rows in
// order, a row's in order.  One workgroup, because rows write behind one another; a wave takes every 16th row, looks at 64 at a time, and
// goes through those that give pages back, once to count them and once, when all that come before are counted, to move them.  Look-ups
// that wait for one another bound it: one row of 32 pages among 16 rows 4.2 us, 16 rows of 128 pages among 256 4.5 us, 100 rows of 32
// pages among 4096 14.6 us (waves that take neighbouring rows 15 and 39.5 us, waves that walk through every row 10.6 and 120).  One row
// of 8192 pages is one wave's: 55 us.
// ---------------------------------------------------------------------------------------------------------
constexpr int kReleaseBlock = 1024;

__global__ __launch_bounds__(kReleaseBlock) void release_kernel(PlaceShape sh, const int32_t *__restrict__ keep, const int32_t *lens, int32_t *table,
                                                                int32_t *free_pages, const int32_t *n_free, int32_t *new_lens, int32_t *n_left)
{
    __shared__ int from[kMaxPagedBatch];                 // pages of a row that go back, then where its first one goes
    __shared__ int sums[kReleaseBlock / 64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int top = min(max(n_free[0], 0), sh.n_pages);
    constexpr int kWaves = kReleaseBlock / 64;           // a wave's rows are b0 + w, b0 + w + 16, ...: rows that end together are often neighbours
    // f(row, its lane, first page that goes back, end of them) for the rows that give any, in order
    auto each_row = [&](int b0, auto f) __attribute__((always_inline)) {
        const int b = b0 + lane * kWaves + w;
        const bool row = b < sh.B;
        const int len = row ? max(lens[b], 0) : 0, kept = row ? min(max(keep[b], 0), len) : 0;
        const int lo = min(blocks_of(sh, (unsigned int)kept), sh.max_blocks), hi = min(blocks_of(sh, (unsigned int)len), sh.max_blocks);
        for (unsigned long long left = __ballot(hi > lo); left != 0ull; left &= left - 1ull) {
            const int r = __ffsll((long long)left) - 1;
            f(b0 + r * kWaves + w, r, __builtin_amdgcn_readlane(lo, r), __builtin_amdgcn_readlane(hi, r));
        }
    };
    for (int b0 = 0; b0 < sh.B; b0 += kReleaseBlock) {
        int mine = 0;
        each_row(b0, [&](int b, int r, int lo, int hi) {
            int n = 0;
            for (int i = lo; i < hi; i += 64) {
                const int p = i + lane < hi ? table[(size_t)b * sh.max_blocks + i + lane] : -1;
                n += __popcll(__ballot((unsigned int)p < (unsigned int)sh.n_pages));
            }
            mine = lane == r ? n : mine;
        });
        const int b = b0 + lane * kWaves + w;
        if (b < sh.B) from[b] = mine;
    }
    __syncthreads();
    // (at most n_pages go back in a table of pages that are in use once; a sum that a broken table makes larger is cut there)
    const int span = (sh.B + kReleaseBlock - 1) / kReleaseBlock, b0 = min(tid * span, sh.B), b1 = min(b0 + span, sh.B);
    const unsigned int cap = (unsigned int)sh.n_pages + 1u;
    unsigned int mine = 0u;
    for (int b = b0; b < b1; ++b) mine = capped(mine, (unsigned int)from[b], cap);
    unsigned int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned int other = (unsigned int)__shfl_up((int)upto, o);
        if (lane >= o) upto = capped(upto, other, cap);
    }
    if (lane == 63) sums[w] = (int)upto;
    unsigned int before = (unsigned int)__shfl_up((int)upto, 1);
    if (lane == 0) before = 0u;
    __syncthreads();
    for (int v = 0; v < w; ++v) before = capped(before, (unsigned int)sums[v], cap);
    for (int b = b0; b < b1; ++b) {
        const unsigned int n = (unsigned int)from[b];
        from[b] = (int)before;
        before = capped(before, n, cap);
    }
    __syncthreads();
    for (int c0 = 0; c0 < sh.B; c0 += kReleaseBlock)
        each_row(c0, [&](int b, int, int lo, int hi) {
            long long at = (long long)top + from[b];
            for (int i = lo; i < hi; i += 64) {
                int32_t *entry = table + (size_t)b * sh.max_blocks + i + lane;
                const int p = i + lane < hi ? *entry : -1;
                const bool page = (unsigned int)p < (unsigned int)sh.n_pages;
                const unsigned long long votes = __ballot(page);
                const long long to = at + __popcll(votes & ((1ull << lane) - 1ull));
                if (page && to < sh.n_pages) free_pages[to] = p;
                if (i + lane < hi) *entry = -1;
                at += __popcll(votes);
            }
        });
    __syncthreads();
    for (int b = tid; b < sh.B; b += kReleaseBlock) new_lens[b] = min(max(keep[b], 0), max(lens[b], 0));
    if (tid == kReleaseBlock - 1) n_left[0] = (int)min((long long)top + before, (long long)sh.n_pages);
}

}  // namespace

size_t place_workspace_bytes(int B) { return ((size_t)B * sizeof(PlacedRow) + 255) / 256 * 256; }

int launch_place_tokens(const PlaceShape &sh, const PlaceIn &in, const PlaceOut &out, void *workspace, hipStream_t stream)
{
    // Up to 1024 rows, a workgroup for every 256 tokens, in one launch; where outputs lie over inputs one workgroup, or two launches of
    // more than 2048 tokens.  Kernel times in us, one workgroup / these / two launches: 16 rows' tokens 3.7; 32 rows, 2000 tokens 8.8 / 5.7; 256 rows
    // with 24 prompts, 26 000 tokens - / 6.6 / 17; 1000 rows, 100 000 tokens - / 8.7 / 18.  (Two launches in a recorded graph take less between
    // them: in place 2.9 and 7.5 us more than one.  One launch would have to wait for all workgroups' reads before the first write.)
    const bool in_place = out.new_lens == in.lens || out.n_left == in.n_free;
    if (sh.B <= 4 * kPlaceBlock && (sh.N <= kPlaceOneTokens || !in_place)) {
        const int workgroups = in_place ? 1 : (sh.N + kPlaceBlock - 1) / kPlaceBlock;
        const dim3 grid((unsigned int)(workgroups < 1 ? 1 : workgroups < kPlaceMost ? workgroups : kPlaceMost));
        return (int)launch_kernel(sh.B <= kPlaceBlock ? place_all_kernel<1> : place_all_kernel<4>, grid, dim3(kPlaceBlock), 0, stream, KernelEvents{}, sh, in, out);
    }
    PlacedRow *rows = static_cast<PlacedRow *>(workspace);
    static_assert(kMaxPagedBatch <= 16 * kPlaceBlock, "rows of a workgroup");
    const hipError_t e = launch_kernel(sh.B <= kPlaceBlock ? place_rows_kernel<1> : place_rows_kernel<16>, dim3(1), dim3(kPlaceBlock), 0, stream, KernelEvents{},
                                       sh, in, out, rows);
    if (e != hipSuccess || sh.N == 0) return (int)e;
    return (int)launch_kernel(place_tokens_kernel, dim3((unsigned int)((sh.N + kPlaceBlock - 1) / kPlaceBlock)), dim3(kPlaceBlock), 0, stream,
                              KernelEvents{}, sh, in, out, rows);
}

int launch_release_pages(const PlaceShape &sh, const int32_t *keep, const int32_t *lens, int32_t *table, int32_t *free_pages,
                         const int32_t *n_free, int32_t *new_lens, int32_t *n_left, hipStream_t stream)
{
    return (int)launch_kernel(release_kernel, dim3(1), dim3(kReleaseBlock), 0, stream, KernelEvents{}, sh, keep, lens, table, free_pages, n_free,
                              new_lens, n_left);
}

}  // namespace chai
