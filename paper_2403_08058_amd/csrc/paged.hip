// Caches in pages: requests of different lengths share one pool of pages, a table names every row's pages in order.  Writing new
// rows into pages (as they are, or as 8-bit codes), attention of one new token per request over its pages, reading pages back.
//
// Method: Sections 2 and 3.4-3.5 as in the contiguous kernels (one score computation per cluster, shared by the members); only
// where a cached row lies is different.  A page holds `page` consecutive positions of every stream: rows [n_pages, streams, page].
#include "chai_rows.h"

#include <hip/hip_ext.h>

#include <type_traits>

namespace chai {

namespace {

constexpr int kWaves = kBlock / 64;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// `workers` waves take at least `least` units each
struct PagedSplit {
    unsigned int workers, least;
};

__device__ __forceinline__ int block_of(const PagedShape &sh, int pos)
{
    return (int)((__umulhi((unsigned int)pos, sh.div_mul) + (unsigned int)pos) >> sh.div_shift);
}

// positions of row b that are attended to
__device__ __forceinline__ int row_len(const PagedShape &sh, int b) { return min(max(sh.lens[b], 0), sh.T_max); }

// ---------------------------------------------------------------------------------------------------------
// How the work of a ragged batch is dealt out.  A unit is one batch of a wave's loads (16 rows of fp32, 32 of bf16, 64 of codes);
// the units of all streams of all rows are laid end to end, (row, stream, unit), and worker w, one wave, takes the quota units from
// w * quota on: every wave streams the same number of bytes whatever the lengths are, which only the device knows.  Each wave adds up
// the rows' units for itself (64 rows per load and six steps of a scan).
// ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned int wave_scan(unsigned int x, int lane)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned int y = (unsigned int)__shfl_up((int)x, o);
        x += lane >= o ? y : 0u;
    }
    return x;
}

template <int U>
struct Deal {
    unsigned int incl, mine;                 // lane l: units of one stream over rows up to and with its own, and of its own rows
    int len;                                 // (up to 64 rows) of the lane's row
    int span;                                // rows per lane
    unsigned int total;                      // units of one stream over all rows

    __device__ __forceinline__ static unsigned int units(int len) { return (unsigned int)(len + U - 1) / U; }

    __device__ __forceinline__ Deal(const PagedShape &sh, int lane)
    {
        span = (sh.B + 63) / 64;
        len = 0;
        mine = 0u;
        for (int i = 0; i < span; ++i) {
            const int b = lane * span + i;
            len = b < sh.B ? row_len(sh, min(b, sh.B - 1)) : 0;
            mine += units(len);
        }
        incl = wave_scan(mine, lane);
        total = (unsigned int)__builtin_amdgcn_readlane((int)incl, 63);
    }

    __device__ __forceinline__ int len_of(const PagedShape &sh, int b) const { return span == 1 ? __builtin_amdgcn_readlane(len, b) : row_len(sh, b); }

    __device__ __forceinline__ unsigned int quota(int streams, const PagedSplit &sp) const
    {
        const unsigned int n = total * (unsigned int)streams;
        return max((n + sp.workers - 1) / sp.workers, sp.least);
    }

    // units of one stream before row b
    __device__ __forceinline__ unsigned int before(const PagedShape &sh, int b, int lane) const
    {
        const int l = b / span;
        unsigned int p = (unsigned int)__builtin_amdgcn_readlane((int)(incl - mine), l);
        if (span > 1) {
            const int r = l * span + lane;
            const unsigned int u = lane < span && r < b ? units(row_len(sh, min(r, sh.B - 1))) : 0u;
            p += (unsigned int)__builtin_amdgcn_readlane((int)wave_scan(u, lane), 63);
        }
        return p;
    }

    // the row that unit y of one stream falls into (y < total), and the units before it
    __device__ __forceinline__ int row_at(const PagedShape &sh, unsigned int y, int lane, unsigned int *first) const
    {
        const int l = __ffsll((long long)__ballot(incl > y)) - 1;
        unsigned int p = (unsigned int)__builtin_amdgcn_readlane((int)(incl - mine), l);
        int b = l * span;
        if (span > 1) {
            const int r = b + lane;
            const unsigned int u = lane < span && r < sh.B ? units(row_len(sh, min(r, sh.B - 1))) : 0u;
            const unsigned int in = wave_scan(u, lane);
            const int i = __ffsll((long long)__ballot(p + in > y)) - 1;
            p += (unsigned int)__builtin_amdgcn_readlane((int)(in - u), i);
            b += i;
        }
        *first = p;
        return b;
    }
};

// The stretches of one stream that a worker's units fall into, one after the other: units ua .. ue-1 of stream s of row b.
template <int U>
struct Walk {
    unsigned int x, x0, x1, ua, ue, n_row, first;        // n_row: units of the stream; first: units of one stream before row b
    int b, s, len;
    __device__ __forceinline__ bool begin(const PagedShape &sh, const Deal<U> &deal, unsigned int worker, int streams, const PagedSplit &sp, int lane)
    {
        const unsigned int quota = deal.quota(streams, sp), n = deal.total * (unsigned int)streams;
        if (worker >= sp.workers || (unsigned long long)worker * quota >= n) return false;
        x = x0 = worker * quota;
        x1 = min(x0 + quota, n);
        b = deal.row_at(sh, x / (unsigned int)streams, lane, &first);
        len = deal.len_of(sh, b);
        n_row = Deal<U>::units(len);
        const unsigned int at = x - first * (unsigned int)streams;
        s = (int)(at / n_row);
        ua = at - (unsigned int)s * n_row;
        ue = min(n_row, ua + (x1 - x));
        return true;
    }
    __device__ __forceinline__ bool next(const PagedShape &sh, const Deal<U> &deal, int streams)
    {
        x += ue - ua;
        if (x >= x1) return false;
        if (++s == streams) {
            s = 0;
            first += n_row;
            do {
                len = deal.len_of(sh, ++b);              // (units are left, so a row is)
                n_row = Deal<U>::units(len);
            } while (n_row == 0u);
        }
        ua = 0;
        ue = min(n_row, x1 - x);
        return true;
    }
    __device__ __forceinline__ bool whole() const { return ua == 0 && ue == n_row; }
    // a worker's parts of streams: the first stretch's, and the last one's where that is another
    __device__ __forceinline__ size_t slot(unsigned int worker) const { return 2 * (size_t)worker + (x == x0 ? 0 : 1); }
};

// Who took a stream of n_row units of which `at` stand before it: `n` workers from `from` on; slot of the i-th one's part.
struct Takers {
    unsigned int from, n, late;
    __device__ __forceinline__ Takers(unsigned int at, unsigned int n_row, unsigned int quota)
    {
        from = at / quota;
        n = (at + n_row - 1) / quota - from + 1;
        late = at != from * quota ? 1u : 0u;
    }
    __device__ __forceinline__ size_t slot(unsigned int i) const { return 2 * (size_t)(from + i) + (i == 0 ? late : 0u); }
};

// ---------------------------------------------------------------------------------------------------------
// Loads of one unit.  A load covers RPW consecutive rows and pages hold multiples of 8, so every load lies in one page: lane i looks up
// the page of load i % 8 and the loads' bases are uniform.  Rows past the end and of absent pages: the pool's first rows are loaded in
// their place, and masked where they are used.
// ---------------------------------------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ int look_up(const PagedShape &sh, const int32_t *table, unsigned int u, unsigned int ue, int len, int lane)
{
    const int row = (int)(u * Tile<DT>::BATCH) + (lane & 7) * Tile<DT>::RPW;
    const int at = table[min(block_of(sh, min(row, sh.T_max - 1)), sh.max_blocks - 1)];
    return u < ue && row < len && (unsigned int)at < (unsigned int)sh.n_pages ? at : -1;
}

// the first row of the lane's load among the pool's rows (0 where there is none)
template <int DT>
__device__ __forceinline__ unsigned int pool_row(const PagedShape &sh, int at, unsigned int u, int streams, int s, int lane)
{
    const int row = (int)(u * Tile<DT>::BATCH) + (lane & 7) * Tile<DT>::RPW;
    return at < 0 ? 0u : (unsigned int)(at * streams + s) * (unsigned int)sh.page + (unsigned int)(row - block_of(sh, row) * sh.page);
}

template <int DT>
__device__ __forceinline__ void request(u32x4 (&buf)[kUnroll], const char *rows, unsigned int row, unsigned int lane_off)
{
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
        buf[i] = stream16(rows + (size_t)(unsigned int)__builtin_amdgcn_readlane((int)row, i) * Tile<DT>::ROW_BYTES + lane_off);
}

// scores of a unit: lane cg < 8 of a lane group gets that of load cg, row rg + cg * RPW of the unit
template <int DT>
__device__ __forceinline__ float dots(const u32x4 (&kb)[kUnroll], const float (&qf)[Tile<DT>::EPL], int cg)
{
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        float f[Tile<DT>::EPL];
        unpack(kb[i], f);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < Tile<DT>::EPL; ++e) dot = fmaf(qf[e], f[e], dot);
        dot = row_sum<DT>(dot);
        mine = cg == i ? dot : mine;
    }
    return mine;
}

// acc += weight * row over a unit's rows; `weight` lies with the lane that owns the row (as in dots), `there` says whether it counts
template <int DT>
__device__ __forceinline__ void weigh(float (&acc)[Tile<DT>::EPL], u32x4 (&vb)[kUnroll], float weight, bool there, float *strip, int cg, int rg)
{
    if (cg < kUnroll) strip[rg * kUnroll + cg] = weight;
    __builtin_amdgcn_wave_barrier();
    float pv[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) pv[i] = strip[rg * kUnroll + i];
    __builtin_amdgcn_wave_barrier();
    if (!__all(there || cg >= kUnroll)) {
        const unsigned long long have = __ballot(there) >> (rg * Tile<DT>::LPR);
#pragma unroll
        for (int i = 0; i < kUnroll; ++i)
            if (!((have >> i) & 1ull)) vb[i] = u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        float f[Tile<DT>::EPL];
        unpack(vb[i], f);
#pragma unroll
        for (int e = 0; e < Tile<DT>::EPL; ++e) acc[e] = fmaf(pv[i], f[e], acc[e]);
    }
}

// the query as the lane multiplies it: elements cg * EPL .. of its representative's row (beside codes q has a type of its own)
template <int DT>
__device__ __forceinline__ void load_query(const char *q, size_t row, int cg, int q_dtype, float (&qf)[Tile<DT>::EPL])
{
    if constexpr (DT == DT_E4M3) {
        const char *p = q + row * (size_t)(kHeadDim * (q_dtype == CHAI_BF16 ? 2 : 4));
        if (q_dtype == CHAI_BF16) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                float f[8];
                unpack(*reinterpret_cast<const u32x4 *>(p + cg * 32 + part * 16), f);
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[part * 8 + e] = f[e];
            }
        } else {
#pragma unroll
            for (int part = 0; part < 4; ++part) {
                float f[4];
                unpack(*reinterpret_cast<const u32x4 *>(p + cg * 64 + part * 16), f);
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[part * 4 + e] = f[e];
            }
        }
    } else {
        unpack(*reinterpret_cast<const u32x4 *>(q + row * Tile<DT>::ROW_BYTES + cg * 16), qf);
    }
}

template <int N>
__device__ __forceinline__ void store_floats(float *p, const float (&f)[N])
{
#pragma unroll
    for (int e = 0; e < N; e += 4) *reinterpret_cast<float4 *>(p + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
}

// the stored score is the rounded product: statistics and probabilities both start from it
template <int DT>
__device__ __forceinline__ float scaled(float dot, float scale, float row_scale)
{
#pragma clang fp contract(off)
    return DT == DT_E4M3 ? (scale * row_scale) * dot : scale * dot;
}

constexpr float kPagedDown = 0x1p-24f;       // times kMaxPagedTokens weights of at most 1: at most 1
constexpr float kPagedLarge = 0x1p120f;

// ---------------------------------------------------------------------------------------------------------
// Attention in one pass: one wave streams keys and values of its units together.  With a running reference m (the largest score so
// far; it moves only when a unit exceeds it, then what has been added up is scaled by exp(old - new)):
//     s[t] = scale * q . K[t],   acc += exp(s[t] - m) V[t],   l += exp(s[t] - m)
// A stream that ends inside the wave's units and began there goes to `out` as acc / l; of others acc / l goes to `partial` and (m, l)
// to `recs` of the wave, two of each (its first units, its last ones), and paged_join_kernel puts them together.
// ---------------------------------------------------------------------------------------------------------
template <int DT, bool IDENT>
__global__ __launch_bounds__(kBlock, DT == DT_E4M3 ? 3 : 4) void paged_attend_kernel(
    PagedShape sh, PagedPages pg, PagedSplit sp, const char *__restrict__ q, int q_dtype, const int32_t *__restrict__ h2c,
    const int32_t *__restrict__ rep, float scale, float *__restrict__ partial, float2 *__restrict__ recs, float *__restrict__ out)
{
    using TL = Tile<DT>;
    constexpr int U = TL::BATCH;
    __shared__ float strip[kWaves][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned int worker = blockIdx.x * kWaves + w;
    const int cg = lane % TL::LPR, rg = lane / TL::LPR;
    const unsigned int lane_off = rg * TL::ROW_BYTES + cg * 16;

    const Deal<U> deal(sh, lane);
    Walk<U> wk;
    if (!wk.begin(sh, deal, worker, sh.H, sp, lane)) return;
    do {
        const int b = wk.b, h = wk.s, len = wk.len;
        const int c = IDENT ? h : min(max(h2c[(size_t)b * sh.H + h], 0), sh.k - 1);
        const int r = IDENT ? h : min(max(rep[(size_t)b * sh.k + c], 0), sh.H - 1);
        const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
        float qf[TL::EPL];
        load_query<DT>(q, (size_t)b * sh.H + r, cg, q_dtype, qf);

        float acc[TL::EPL], m_ref, l_run, down = 1.f;
        for (;;) {
            u32x4 kb[kUnroll], vb[kUnroll];
            float ks = 1.f, vs = 1.f;
            int at = look_up<DT>(sh, table, wk.ua, wk.ue, len, lane), at1 = look_up<DT>(sh, table, wk.ua + 1, wk.ue, len, lane);
            unsigned int krow = pool_row<DT>(sh, at, wk.ua, sh.k, c, lane), vrow = pool_row<DT>(sh, at, wk.ua, sh.H, h, lane);
            request<DT>(kb, pg.k, krow, lane_off);
            if (DT == DT_E4M3) ks = pg.k_scales[krow + (at < 0 ? 0 : rg)];
            request<DT>(vb, pg.v, vrow, lane_off);
            if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at < 0 ? 0 : rg)];
#pragma unroll
            for (int e = 0; e < TL::EPL; ++e) acc[e] = 0.f;
            m_ref = -INFINITY;
            l_run = 0.f;
            for (unsigned int u = wk.ua; u < wk.ue; ++u) {
                const int at2 = look_up<DT>(sh, table, u + 2, wk.ue, len, lane);
                const float mine = dots<DT>(kb, qf, cg);
                const bool there = cg < kUnroll && at >= 0 && (int)(u * U) + cg * TL::RPW + rg < len;
                const float sv = there ? scaled<DT>(mine, scale, ks) : -INFINITY;
                krow = pool_row<DT>(sh, at1, u + 1, sh.k, c, lane);
                request<DT>(kb, pg.k, krow, lane_off);
                if (DT == DT_E4M3) ks = pg.k_scales[krow + (at1 < 0 ? 0 : rg)];
                if (__any(sv > m_ref)) {
                    const float m_new = fmaxf(m_ref, wave_max(sv));
                    const float f = __expf(m_ref - m_new);
#pragma unroll
                    for (int e = 0; e < TL::EPL; ++e) acc[e] *= f;
                    l_run *= f;
                    m_ref = m_new;
                }
                const float p = __expf(sv - (m_ref == -INFINITY ? 0.f : m_ref)) * down;
                l_run += p;
                weigh<DT>(acc, vb, DT == DT_E4M3 ? (there ? p * vs : 0.f) : p, there, strip[w], cg, rg);
                vrow = pool_row<DT>(sh, at1, u + 1, sh.H, h, lane);
                request<DT>(vb, pg.v, vrow, lane_off);
                if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at1 < 0 ? 0 : rg)];
                at = at1;
                at1 = at2;
            }
            // lane groups; sums beyond the largest float (the quotient is not) are taken again with smaller weights
            bool large = false;
#pragma unroll
            for (int e = 0; e < TL::EPL; ++e) {
#pragma unroll
                for (int o = TL::LPR; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o);
                large = large || !(fabsf(acc[e]) <= kPagedLarge);
            }
            if (!__any(large) || down != 1.f) break;
            down = kPagedDown;
        }
        const float l = wave_sum(l_run);
#pragma unroll
        for (int e = 0; e < TL::EPL; ++e) acc[e] = l == 0.f ? 0.f : acc[e] / l;
        if (wk.whole()) {
            if (rg == 0) store_floats(out + ((size_t)b * sh.H + h) * kHeadDim + cg * TL::EPL, acc);
        } else {
            const size_t slot = wk.slot(worker);
            if (rg == 0) store_floats(partial + slot * kHeadDim + cg * TL::EPL, acc);
            if (lane == 0) recs[slot] = make_float2(m_ref, l / down);
        }
    } while (wk.next(sh, deal, sh.H));
}

// ---------------------------------------------------------------------------------------------------------
// Attention in two passes, for layers with fewer clusters than heads: the keys of a cluster are read once, not once per member.
// Scores: a wave streams keys of its units, writes s[b][j][t] (-inf where nothing is to be attended to, whole units) and the maximum
// and sum of exponentials of every stretch: `whole` of a stream that it took alone, else `parts` of the wave.
// ---------------------------------------------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(kBlock, DT == DT_E4M3 ? 5 : 6) void paged_scores_kernel(PagedShape sh, PagedPages pg, PagedSplit sp, const char *__restrict__ q,
                                                                 int q_dtype, const int32_t *__restrict__ rep, float scale, int T_pad,
                                                                 float *__restrict__ scores, float2 *__restrict__ whole,
                                                                 float2 *__restrict__ parts)
{
    using TL = Tile<DT>;
    constexpr int U = TL::BATCH;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned int worker = blockIdx.x * kWaves + w;
    const int cg = lane % TL::LPR, rg = lane / TL::LPR;
    const unsigned int lane_off = rg * TL::ROW_BYTES + cg * 16;

    const Deal<U> deal(sh, lane);
    Walk<U> wk;
    if (!wk.begin(sh, deal, worker, sh.k, sp, lane)) return;
    do {
        const int b = wk.b, j = wk.s, len = wk.len;
        const int r = min(max(rep[(size_t)b * sh.k + j], 0), sh.H - 1);
        const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
        u32x4 kb[kUnroll];
        float ks = 1.f;
        int at = look_up<DT>(sh, table, wk.ua, wk.ue, len, lane), at1 = look_up<DT>(sh, table, wk.ua + 1, wk.ue, len, lane);
        unsigned int krow = pool_row<DT>(sh, at, wk.ua, sh.k, j, lane);
        request<DT>(kb, pg.k, krow, lane_off);
        if (DT == DT_E4M3) ks = pg.k_scales[krow + (at < 0 ? 0 : rg)];
        float qf[TL::EPL];
        load_query<DT>(q, (size_t)b * sh.H + r, cg, q_dtype, qf);
        float *srow = scores + ((size_t)b * sh.k + j) * T_pad;
        float m_run = -INFINITY, l_run = 0.f;            // of the scores that this lane has seen
        for (unsigned int u = wk.ua; u < wk.ue; ++u) {
            const int at2 = look_up<DT>(sh, table, u + 2, wk.ue, len, lane);
            const float mine = dots<DT>(kb, qf, cg);
            const int t = (int)(u * U) + cg * TL::RPW + rg;
            const bool there = cg < kUnroll && at >= 0 && t < len;
            const float sv = there ? scaled<DT>(mine, scale, ks) : -INFINITY;
            krow = pool_row<DT>(sh, at1, u + 1, sh.k, j, lane);
            request<DT>(kb, pg.k, krow, lane_off);
            if (DT == DT_E4M3) ks = pg.k_scales[krow + (at1 < 0 ? 0 : rg)];
            if (cg < kUnroll) srow[t] = sv;
            const float m_new = fmaxf(m_run, sv), ref = m_new == -INFINITY ? 0.f : m_new;
            l_run = l_run * __expf(m_run - ref) + __expf(sv - ref);
            m_run = m_new;
            at = at1;
            at1 = at2;
        }
        const float M = wave_max(m_run);
        const float L = wave_sum(m_run == -INFINITY ? l_run : l_run * __expf(m_run - M));     // (lanes that saw only NaN hold it in l_run)
        if (lane == 0) (wk.whole() ? whole[(size_t)b * sh.k + j] : parts[wk.slot(worker)]) = make_float2(M, L);
    } while (wk.next(sh, deal, sh.k));
}

// Maximum and sum of exponentials over a stream's parts.
__device__ __forceinline__ float2 merge(const float2 *parts, const Takers &tk, int lane)
{
    float m = -INFINITY;
    for (unsigned int i = lane; i < tk.n; i += 64) m = fmaxf(m, parts[tk.slot(i)].x);
    const float M = wave_max(m);
    float l = 0.f;
    for (unsigned int i = lane; i < tk.n; i += 64) {
        const float2 rc = parts[tk.slot(i)];
        l += rc.x == -INFINITY ? rc.y : rc.y * __expf(rc.x - M);         // (only -inf scores: 0, NaN among them: NaN)
    }
    return make_float2(M, wave_sum(l));
}

// Values: a wave streams the values of its units, each weighed by its cluster's probability exp(s - M) / L.
template <int DT>
__global__ __launch_bounds__(kBlock, DT == DT_F32 ? 6 : (DT == DT_BF16 ? 5 : 4)) void paged_values_kernel(PagedShape sh, PagedPages pg, PagedSplit sp, PagedSplit sp_scores,
                                                                 const int32_t *__restrict__ h2c, int T_pad,
                                                                 const float *__restrict__ scores, const float2 *__restrict__ whole,
                                                                 const float2 *__restrict__ parts, float *__restrict__ partial,
                                                                 float *__restrict__ out)
{
    using TL = Tile<DT>;
    constexpr int U = TL::BATCH;
    __shared__ float strip[kWaves][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned int worker = blockIdx.x * kWaves + w;
    const int cg = lane % TL::LPR, rg = lane / TL::LPR;
    const unsigned int lane_off = rg * TL::ROW_BYTES + cg * 16;

    const Deal<U> deal(sh, lane);
    Walk<U> wk;
    if (!wk.begin(sh, deal, worker, sh.H, sp, lane)) return;
    do {
        const int b = wk.b, h = wk.s, len = wk.len;
        const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
        const int c = min(max(h2c[(size_t)b * sh.H + h], 0), sh.k - 1);
        u32x4 vb[kUnroll];
        float vs = 1.f;
        int at = look_up<DT>(sh, table, wk.ua, wk.ue, len, lane), at1 = look_up<DT>(sh, table, wk.ua + 1, wk.ue, len, lane);
        unsigned int vrow = pool_row<DT>(sh, at, wk.ua, sh.H, h, lane);
        request<DT>(vb, pg.v, vrow, lane_off);
        if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at < 0 ? 0 : rg)];
        const float *srow = scores + ((size_t)b * sh.k + c) * T_pad + (cg < kUnroll ? cg * TL::RPW + rg : 0);
        float sv = srow[wk.ua * U];
        const Takers tk(wk.first * (unsigned int)sh.k + (unsigned int)c * wk.n_row, wk.n_row, deal.quota(sh.k, sp_scores));
        const float2 st = tk.n == 1 ? whole[(size_t)b * sh.k + c] : merge(parts, tk, lane);
        const float M = st.x == -INFINITY ? 0.f : st.x, inv = st.y == 0.f ? 0.f : 1.f / st.y;
        float acc[TL::EPL];
#pragma unroll
        for (int e = 0; e < TL::EPL; ++e) acc[e] = 0.f;
        for (unsigned int u = wk.ua; u < wk.ue; ++u) {
            const int at2 = look_up<DT>(sh, table, u + 2, wk.ue, len, lane);
            const bool there = cg < kUnroll && at >= 0 && (int)(u * U) + cg * TL::RPW + rg < len;
            const float p = there ? __expf(sv - M) * inv : 0.f;
            weigh<DT>(acc, vb, DT == DT_E4M3 ? (there ? p * vs : 0.f) : p, there, strip[w], cg, rg);
            vrow = pool_row<DT>(sh, at1, u + 1, sh.H, h, lane);
            request<DT>(vb, pg.v, vrow, lane_off);
            if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at1 < 0 ? 0 : rg)];
            sv = srow[min(u + 1, wk.ue - 1) * U];
            at = at1;
            at1 = at2;
        }
#pragma unroll
        for (int e = 0; e < TL::EPL; ++e) {
#pragma unroll
            for (int o = TL::LPR; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o);
        }
        float *o = wk.whole() ? out + ((size_t)b * sh.H + h) * kHeadDim : partial + wk.slot(worker) * kHeadDim;
        if (rg == 0) store_floats(o + cg * TL::EPL, acc);
    } while (wk.next(sh, deal, sh.H));
}

// Streams that several waves took.  WEIGHED (one pass): out = mean of their parts, each weighed by its sum of exponentials times
// exp(its reference - the largest); else their sum.  A wave per (row, head), two columns per lane; streams that one wave took are left
// alone, rows without a position get 0.
template <int U, bool WEIGHED>
__global__ __launch_bounds__(kBlock) void paged_join_kernel(PagedShape sh, PagedSplit sp, const float *__restrict__ partial,
                                                            const float2 *__restrict__ recs, float *__restrict__ out)
{
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x * kWaves + w, b = blockIdx.y;
    if (h >= sh.H) return;
    float2 *o = reinterpret_cast<float2 *>(out + ((size_t)b * sh.H + h) * kHeadDim) + lane;
    const Deal<U> deal(sh, lane);
    const unsigned int n_row = Deal<U>::units(deal.len_of(sh, b));
    if (n_row == 0u) {
        *o = make_float2(0.f, 0.f);
        return;
    }
    const Takers tk(deal.before(sh, b, lane) * (unsigned int)sh.H + (unsigned int)h * n_row, n_row, deal.quota(sh.H, sp));
    if (tk.n == 1) return;
    float2 st = make_float2(0.f, 1.f);
    if (WEIGHED) st = merge(recs, tk, lane);
    const float inv = st.y == 0.f ? 0.f : 1.f / st.y;
    float2 sum = make_float2(0.f, 0.f);
    for (unsigned int i0 = 0; i0 < tk.n; i0 += 64) {
        float wt = 0.f;
        if (WEIGHED && i0 + lane < tk.n) {
            const float2 rc = recs[tk.slot(i0 + lane)];
            wt = (rc.x == -INFINITY ? rc.y : rc.y * __expf(rc.x - st.x)) * inv;
        }
        const unsigned int here = min(tk.n - i0, 64u);
        for (unsigned int i = 0; i < here; i += 8) {
            float2 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = reinterpret_cast<const float2 *>(partial + tk.slot(i0 + min(i + j, here - 1)) * kHeadDim)[lane];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float wj = WEIGHED ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), (int)min(i + j, 63u))) : 1.f;
                if (i + j < here) {
                    sum.x = fmaf(wj, v[j].x, sum.x);
                    sum.y = fmaf(wj, v[j].y, sum.y);
                }
            }
        }
    }
    *o = sum;
}

// ---------------------------------------------------------------------------------------------------------
// New rows into pages, and pages into contiguous rows.  A workgroup takes `rows` rows of one request: 1 << shift consecutive tokens (so
// that one new token of many streams fills a workgroup as well) of rows >> shift streams; streams are the k key slots, then the H value
// heads.  Sixteen lanes per row, eight elements each, all rows requested at once.
// ---------------------------------------------------------------------------------------------------------
template <bool BF16>
constexpr int kMoveUnroll = BF16 ? 8 : 4;
constexpr int move_rows(bool bf16) { return kBlock / 16 * (bf16 ? kMoveUnroll<true> : kMoveUnroll<false>); }

// Where a wave's rows are and go, one row per lane: row r of a wave is that of its lane group r % 4 (sixteen lanes) in round r / 4, and
// the sixteen lanes of the group fetch it from lane r.  (Looked up by every lane for itself the multiplications took longer than the
// rows: 16 x 40 streams of up to 2043 tokens quantised 79.7 us.)
struct Places {
    unsigned int at;                         // row among the pool's rows of its kind, kNowhere: in no page
    unsigned int lo, hi;                     // the other side: 64 bits of offset below kIsKey, or a row
};
constexpr unsigned int kNowhere = 0xffffffffu, kIsKey = 0x80000000u;

template <bool BF16, typename Other>
__device__ __forceinline__ Places find_places(const PagedShape &sh, const int32_t *start, const int32_t *count, int Tn, int shift, int lane, int w, Other other)
{
    const int b = blockIdx.z;
    Places pl = {kNowhere, kNowhere, 0u};
    int n = Tn, first;
    if (start == nullptr) {                  // the last position of every row
        first = sh.lens[b] - 1;
        n = first >= 0 && first < sh.T_max ? 1 : 0;
    } else {
        first = start[b];
        if (count != nullptr) n = min(max(count[b], 0), Tn);
    }
    const int local = (lane / 4) * (kBlock / 16) + w * 4 + lane % 4;
    const int token = (int)(blockIdx.x << shift) + (local & ((1 << shift) - 1));
    const int stream = blockIdx.y * (move_rows(BF16) >> shift) + (local >> shift);
    if (lane < 4 * kMoveUnroll<BF16> && token < n && stream < sh.k + sh.H) {
        const int pos = (int)((unsigned int)first + (unsigned int)token), block = block_of(sh, max(pos, 0));
        const bool key = stream < sh.k;
        const int streams = key ? sh.k : sh.H, s = key ? stream : stream - sh.k;
        const int page_at = pos >= 0 && block < sh.max_blocks ? sh.table[(size_t)b * sh.max_blocks + block] : -1;
        if ((unsigned int)page_at < (unsigned int)sh.n_pages)
            pl.at = (unsigned int)(page_at * streams + s) * (unsigned int)sh.page + (unsigned int)(pos - block * sh.page);
        other(pl, b, key, s, token);
    }
    return pl;
}

// a lane's eight elements of a row as they are held: one 16-byte word of bf16, two of fp32
template <bool BF16>
struct RawPiece {
    u32x4 x[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const char *row, int piece)
    {
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) x[i] = stream16(row + piece * (BF16 ? 16 : 32) + i * 16);
    }
    __device__ __forceinline__ void store(char *row, int piece) const
    {
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4 *>(row + piece * (BF16 ? 16 : 32) + i * 16));
    }
    __device__ __forceinline__ Piece widened() const
    {
        Piece p;
        if constexpr (BF16) {
            unpack(x[0], p.x);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p.x[e] = __uint_as_float(x[e / 4][e % 4]);
        }
        return p;
    }
    __device__ __forceinline__ void set(const float (&f)[8])
    {
        if constexpr (BF16) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[0][e] = __builtin_bit_cast(unsigned int, __builtin_convertvector(f32x2{f[2 * e], f[2 * e + 1]}, bf16x2));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e / 4][e % 4] = __float_as_uint(f[e]);
        }
    }
};

template <int DT, bool BF16>
__global__ __launch_bounds__(kBlock) void paged_append_kernel(PagedShape sh, PagedPages pg, const char *__restrict__ k_new,
                                                              const char *__restrict__ v_new, long long k_stride, long long v_stride,
                                                              const int32_t *__restrict__ rep, const int32_t *__restrict__ start,
                                                              const int32_t *__restrict__ count, int Tn, int shift)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, piece = lane & 15, rg = lane >> 4;
    constexpr int kBytes = BF16 ? 2 : 4, N = kMoveUnroll<BF16>;
    const Places pl = find_places<BF16>(sh, start, count, Tn, shift, lane, w, [&](Places &x, int b, bool key, int s, int token) {
        const int h = key && rep != nullptr ? min(rep[(size_t)b * sh.k + s], sh.H - 1) : s;
        if (h < 0) x.at = kNowhere;          // (a slot without a cluster keeps what it holds)
        const unsigned long long from = (((unsigned long long)b * sh.H + max(h, 0)) * (key ? k_stride : v_stride) + (unsigned long long)token * kHeadDim) * kBytes;
        x.lo = (unsigned int)from;
        x.hi = (unsigned int)(from >> 32) | (key ? kIsKey : 0u);
    });
    if (!__any(pl.at != kNowhere)) return;
    unsigned int at[N];
    bool key[N];
    RawPiece<BF16> p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = i * 4 + rg;
        at[i] = (unsigned int)__shfl((int)pl.at, r);
        const unsigned int lo = (unsigned int)__shfl((int)pl.lo, r), hi = (unsigned int)__shfl((int)pl.hi, r);
        key[i] = (hi & kIsKey) != 0u;
        if (at[i] != kNowhere) p[i].load((key[i] ? k_new : v_new) + (((unsigned long long)(hi & ~kIsKey) << 32) | lo), piece);
    }
    if constexpr (DT == DT_E4M3) {
        // lane i of a group turns the largest value of the group's row i into its scale and factor, then hands the factor on
        float amax[N], mine = 0.f;
        unsigned int mine_at = kNowhere;
        bool mine_key = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            amax[i] = largest_of(p[i].widened());
            mine = piece == i ? amax[i] : mine;
            mine_at = piece == i ? at[i] : mine_at;
            mine_key = piece == i ? key[i] : mine_key;
        }
        const float factor = 448.0f / mine;
        if (mine_at != kNowhere) const_cast<float *>(mine_key ? pg.k_scales : pg.v_scales)[mine_at] = mine == 0.f ? 0.f : mine / 448.0f;
        auto write = [&](auto self, auto index) {
            constexpr int i = decltype(index)::value;
            const float inv = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(factor), 0x150 + i, 0xf, 0xf, false));     // row_newbcast: lane i
            if (at[i] != kNowhere) {
                const uint2 codes = codes_of(p[i].widened(), inv);
                reinterpret_cast<uint2 *>(const_cast<char *>(key[i] ? pg.k : pg.v))[(size_t)at[i] * 16 + piece] = amax[i] == 0.f ? make_uint2(0u, 0u) : codes;
            }
            if constexpr (i + 1 < N) self(self, std::integral_constant<int, i + 1>{});
        };
        write(write, std::integral_constant<int, 0>{});
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at[i] != kNowhere) p[i].store(const_cast<char *>(key[i] ? pg.k : pg.v) + (size_t)at[i] * (kHeadDim * kBytes), piece);
    }
}

template <int DT, bool BF16>
__global__ __launch_bounds__(kBlock) void paged_gather_kernel(PagedShape sh, PagedPages pg, const int32_t *__restrict__ start,
                                                              const int32_t *__restrict__ count, char *__restrict__ k_out,
                                                              char *__restrict__ v_out, int Tn, int shift)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, piece = lane & 15, rg = lane >> 4;
    constexpr int kBytes = BF16 ? 2 : 4, N = kMoveUnroll<BF16>;
    const Places pl = find_places<BF16>(sh, start, count, Tn, shift, lane, w, [&](Places &x, int b, bool key, int s, int token) {
        x.lo = (unsigned int)((b * (key ? sh.k : sh.H) + s) * (long long)Tn + token);        // (row of an output of 256 bytes and more a row)
        x.hi = key ? kIsKey : 0u;
    });
    if (!__any(pl.lo != kNowhere)) return;
    unsigned int at[N], to[N];
    bool key[N];
    RawPiece<BF16> p[N];
    u32x2 codes[N];
    float scale[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = i * 4 + rg;
        at[i] = (unsigned int)__shfl((int)pl.at, r);
        to[i] = (unsigned int)__shfl((int)pl.lo, r);
        key[i] = __shfl((int)pl.hi, r) != 0;
        if (at[i] == kNowhere) continue;
        const char *rows = key[i] ? pg.k : pg.v;
        if constexpr (DT == DT_E4M3) {
            codes[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(rows) + (size_t)at[i] * 16 + piece);
            scale[i] = (key[i] ? pg.k_scales : pg.v_scales)[at[i]];
        } else {
            p[i].load(rows + (size_t)at[i] * (kHeadDim * kBytes), piece);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (to[i] == kNowhere) continue;
        if (at[i] == kNowhere) {
#pragma unroll
            for (auto &x : p[i].x) x = u32x4{0u, 0u, 0u, 0u};
        } else if constexpr (DT == DT_E4M3) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i][e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i][e], true);
                f[4 * e] = lo.x * scale[i];
                f[4 * e + 1] = lo.y * scale[i];
                f[4 * e + 2] = hi.x * scale[i];
                f[4 * e + 3] = hi.y * scale[i];
            }
            p[i].set(f);
        }
        p[i].store((key[i] ? k_out : v_out) + (size_t)to[i] * (kHeadDim * kBytes), piece);
    }
}

// tokens per workgroup, as a power of two: all of them up to `rows`
int move_shift(int Tn, int rows)
{
    int shift = 0;
    while ((1 << shift) < Tn && (1 << shift) < rows) ++shift;
    return shift;
}

dim3 move_grid(const PagedShape &sh, int Tn, int shift, int rows)
{
    const int streams = rows >> shift;
    return dim3((unsigned int)((Tn + (1 << shift) - 1) >> shift), (unsigned int)((sh.k + sh.H + streams - 1) / streams), (unsigned int)sh.B);
}

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int unit_rows(int cache_dtype) { return cache_dtype == CHAI_F32 ? Tile<DT_F32>::BATCH : (cache_dtype == CHAI_BF16 ? Tile<DT_BF16>::BATCH : Tile<DT_E4M3>::BATCH); }

}  // namespace

// Waves of a launch.  Of the two passes, which have one stream of loads each, in us for 1024 / 2048 / 3072 / 4096 / 6144 to 8192:
// scores of 64 x 8 rows of codes (4096 tokens at most, most short) 23.1 / 17.2 / 16.6 / 16.2 / 16.5 and values of 64 x 32 - / 49 / 45
// / 41.6 / 44.6; 4 x 32 of 32768 bf16 tokens within 2 % up to 4096, 173 / 163 with 8192.  One pass has keys and values in flight: 8 x
// 52 heads of up to 1777 bf16 tokens 37.4 / 36.4 / 41 / 43.6 / 42.
constexpr unsigned int kStreamWorkers = 4096, kAttendWorkers = 2048, kPagedWorkers = 4096;
constexpr unsigned int kPagedParts = 64;               // most waves of one stream

static int padded_tokens(int T_max) { return (T_max + 63) / 64 * 64; }

PagedPlan make_paged_plan(int B, int H, int k, int T_max)
{
    PagedPlan pl;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    pl.off_recs = take(2 * (size_t)kPagedWorkers * sizeof(float2));
    pl.off_partial = take(2 * (size_t)kPagedWorkers * kHeadDim * sizeof(float));
    pl.off_whole = take((size_t)B * k * sizeof(float2));
    pl.off_scores = take((size_t)B * k * padded_tokens(T_max) * sizeof(float));
    pl.bytes = off;
    return pl;
}

static PagedSplit make_paged_split(int B, int streams, int T_max, int cache_dtype, unsigned int workers)
{
    PagedSplit sp;
    const int u = unit_rows(cache_dtype);
    const long long row_units = ((long long)T_max + u - 1) / u, units = row_units * B * streams;
    sp.workers = (unsigned int)(units < (long long)workers ? units : workers);
    sp.least = (unsigned int)((row_units + kPagedParts - 1) / kPagedParts);
    return sp;
}

void set_page_division(PagedShape *sh)
{
    // floor(n / page) = (mulhi(n, mul) + n) >> shift for every 0 <= n < 2^31
    int s = 0;
    while ((1ll << s) < sh->page) ++s;
    sh->div_shift = s;
    sh->div_mul = (unsigned int)((((1ull << s) - (unsigned long long)sh->page) << 32) / (unsigned long long)sh->page + 1ull);
}

template <int DT>
static int paged_attention_typed(const PagedShape &sh, const PagedPages &pg, const char *q, int dtype, const int32_t *h2c, const int32_t *rep,
                                 float scale, float *out, char *ws, const PagedPlan &plan, hipStream_t stream)
{
    constexpr int U = Tile<DT>::BATCH, cache = DT;
    float2 *recs = reinterpret_cast<float2 *>(ws + plan.off_recs), *whole = reinterpret_cast<float2 *>(ws + plan.off_whole);
    float *partial = reinterpret_cast<float *>(ws + plan.off_partial), *scores = reinterpret_cast<float *>(ws + plan.off_scores);
    const dim3 block(kBlock), heads((unsigned int)(sh.H + kWaves - 1) / kWaves, (unsigned int)sh.B);
    auto waves = [](const PagedSplit &sp) { return dim3((sp.workers + kWaves - 1) / kWaves); };
    const KernelEvents none;
    if (h2c == nullptr) {
        const PagedSplit sp = make_paged_split(sh.B, sh.H, sh.T_max, cache, kAttendWorkers);
        const hipError_t e = launch_kernel(paged_attend_kernel<DT, true>, waves(sp), block, 0, stream,
                                           none, sh, pg, sp, q, dtype, h2c, rep, scale, partial, recs, out);
        if (e != hipSuccess) return (int)e;
        return (int)launch_kernel(paged_join_kernel<U, true>, heads, block, 0, stream, none, sh, sp, partial, recs, out);
    }
    const PagedSplit ss = make_paged_split(sh.B, sh.k, sh.T_max, cache, kStreamWorkers), sv = make_paged_split(sh.B, sh.H, sh.T_max, cache, kStreamWorkers);
    const int T_pad = padded_tokens(sh.T_max);
    hipError_t e = launch_kernel(paged_scores_kernel<DT>, waves(ss), block, 0, stream, none, sh, pg, ss, q, dtype, rep, scale, T_pad, scores, whole, recs);
    if (e != hipSuccess) return (int)e;
    e = launch_kernel(paged_values_kernel<DT>, waves(sv), block, 0, stream, none, sh, pg, sv, ss, h2c, T_pad, scores, whole, recs, partial, out);
    if (e != hipSuccess) return (int)e;
    return (int)launch_kernel(paged_join_kernel<U, false>, heads, block, 0, stream, none, sh, sv, partial, nullptr, out);
}

int launch_paged_attention(const PagedShape &sh, const PagedPages &pg, const void *q, int dtype, int cache_dtype, const int32_t *h2c,
                           const int32_t *rep, float scale, float *out, void *workspace, const PagedPlan &plan, hipStream_t stream)
{
    auto *typed = cache_dtype == CHAI_F32 ? paged_attention_typed<DT_F32> : (cache_dtype == CHAI_BF16 ? paged_attention_typed<DT_BF16> : paged_attention_typed<DT_E4M3>);
    return typed(sh, pg, static_cast<const char *>(q), dtype, h2c, rep, scale, out, static_cast<char *>(workspace), plan, stream);
}

int launch_paged_append(const PagedShape &sh, const PagedPages &pg, const void *k_new, const void *v_new, int64_t k_stride,
                        int64_t v_stride, const int32_t *rep, const int32_t *start, const int32_t *count, int Tn, int dtype,
                        int cache_dtype, hipStream_t stream)
{
    const int rows = move_rows(dtype == CHAI_BF16), shift = move_shift(Tn, rows);
    const char *kc = static_cast<const char *>(k_new), *vc = static_cast<const char *>(v_new);
    auto go = [&](auto *kernel) {
        return (int)launch_kernel(kernel, move_grid(sh, Tn, shift, rows), dim3(kBlock), 0, stream, KernelEvents(), sh, pg, kc, vc, k_stride, v_stride,
                                  rep, start, count, Tn, shift);
    };
    if (cache_dtype == CHAI_E4M3) return dtype == CHAI_BF16 ? go(paged_append_kernel<DT_E4M3, true>) : go(paged_append_kernel<DT_E4M3, false>);
    return dtype == CHAI_BF16 ? go(paged_append_kernel<DT_BF16, true>) : go(paged_append_kernel<DT_F32, false>);
}

int launch_paged_gather(const PagedShape &sh, const PagedPages &pg, const int32_t *start, const int32_t *count, void *k_out, void *v_out,
                        int Tn, int dtype, int cache_dtype, hipStream_t stream)
{
    const int rows = move_rows(dtype == CHAI_BF16), shift = move_shift(Tn, rows);
    char *ko = static_cast<char *>(k_out), *vo = static_cast<char *>(v_out);
    auto go = [&](auto *kernel) {
        return (int)launch_kernel(kernel, move_grid(sh, Tn, shift, rows), dim3(kBlock), 0, stream, KernelEvents(), sh, pg, start, count, ko, vo, Tn,
                                  shift);
    };
    if (cache_dtype == CHAI_E4M3) return dtype == CHAI_BF16 ? go(paged_gather_kernel<DT_E4M3, true>) : go(paged_gather_kernel<DT_E4M3, false>);
    return dtype == CHAI_BF16 ? go(paged_gather_kernel<DT_BF16, true>) : go(paged_gather_kernel<DT_F32, false>);
}

}  // namespace chai
