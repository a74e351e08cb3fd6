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

// n / d without a division, for 0 <= n < 2^31: (mulhi(n, mul) + n) >> shift
struct Quotient {
    unsigned int mul;
    int shift;
};
// 1 << shift waves take at least `least` units each of `streams` streams a row; both go by the bound of the lengths (make_paged_split)
struct PagedSplit {
    int shift;
    unsigned int least;
    Quotient by_streams;
};
inline unsigned int workers_of(const PagedSplit &sp) { return 1u << sp.shift; }

__device__ __forceinline__ int block_of(const PagedShape &sh, int pos)
{
    return (int)((__umulhi((unsigned int)pos, sh.div_mul) + (unsigned int)pos) >> sh.div_shift);
}

// Sums and maxima over a wave without the LDS crossbar (six steps of it are some 600 cycles in a row): DPP within sixteen lanes, then the
// four rows of them; on two halves or rows at once a swap leaves both partners in both places.
__device__ __forceinline__ float rows_of_lane(float x, int row) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), row * 16)); }

__device__ __forceinline__ float all_max(float x)
{
    x = dpp_max<0xB1>(x);                    // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
    x = dpp_max<0x4E>(x);
    x = dpp_max<0x141>(x);
    x = dpp_max<0x140>(x);
    return fmaxf(fmaxf(rows_of_lane(x, 0), rows_of_lane(x, 1)), fmaxf(rows_of_lane(x, 2), rows_of_lane(x, 3)));
}

__device__ __forceinline__ float all_sum(float x)
{
    x = dpp_add<0xB1>(x);
    x = dpp_add<0x4E>(x);
    x = dpp_add<0x141>(x);
    x = dpp_add<0x140>(x);
    return (rows_of_lane(x, 0) + rows_of_lane(x, 1)) + (rows_of_lane(x, 2) + rows_of_lane(x, 3));
}

// sum over the lane groups of a wave, LPR lanes each, in every lane
template <int LPR>
__device__ __forceinline__ float sum_groups(float x)
{
    typedef unsigned int pair __attribute__((ext_vector_type(2)));
    if (LPR == 8) x = dpp_add<0x128>(x);     // row_ror:8
    if (LPR <= 16) {
        const pair y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(y.x) + __uint_as_float(y.y);
    }
    const pair y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(y.x) + __uint_as_float(y.y);
}

// positions of a row that are attended to
__device__ __forceinline__ int taken_len(const PagedShape &sh, int given) { return min(max(given, 0), sh.T_max); }
__device__ __forceinline__ int given_of(const PagedShape &sh, int b) { return sh.lens != nullptr ? sh.lens[b] : sh.T_max; }
__device__ __forceinline__ int row_len(const PagedShape &sh, int b) { return taken_len(sh, given_of(sh, b)); }

// ---------------------------------------------------------------------------------------------------------
// How the work of a ragged batch is dealt out.  A unit is one batch of a wave's loads (16 rows of fp32, 32 of bf16, 64 of codes);
// the units of all streams of all rows are laid end to end, (row, stream, unit), and worker w, one wave, takes the quota units from
// w * quota on: waves that have work stream the same number of bytes whatever the lengths are, which only the device knows.  How many
// have work goes by the bound as well: a share is at least 1 / 32 of a row at the bound (1 / 128 of its scores), so a bound far above the rows
// leaves waves without any.  Each wave adds up the rows' units for itself (64 rows per load and six steps of a scan).
// ---------------------------------------------------------------------------------------------------------
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned int add_from(unsigned int x)
{
    return x + (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
// sums over lanes 0 .. l
__device__ __forceinline__ unsigned int wave_scan(unsigned int x)
{
    x = add_from<0x111, 0xf>(x);             // row_shr:1, :2, :4, :8
    x = add_from<0x112, 0xf>(x);
    x = add_from<0x114, 0xf>(x);
    x = add_from<0x118, 0xf>(x);
    x = add_from<0x142, 0xa>(x);             // the last lane of rows 0 and 2 to rows 1 and 3, that of the lower half to the upper one
    return add_from<0x143, 0xc>(x);
}

template <int U>
struct Deal {
    unsigned int incl, mine;                 // lane l: units of one stream over rows up to and with its own, and of its own rows
    int given;                               // (up to 64 rows) seq_lens of the lane's row
    int span;                                // rows per lane
    unsigned int total;                      // units of one stream over all rows

    __device__ __forceinline__ static unsigned int units(int len) { return (unsigned int)(len + U - 1) / U; }

    __device__ __forceinline__ Deal(const PagedShape &sh, int lane)
    {
        span = (sh.B + 63) / 64;
        given = 0;
        mine = 0u;
        for (int i = 0; i < span; ++i) {
            const int b = lane * span + i;
            given = b < sh.B ? given_of(sh, min(b, sh.B - 1)) : 0;
            mine += units(taken_len(sh, given));
        }
        incl = wave_scan(mine);
        total = (unsigned int)__builtin_amdgcn_readlane((int)incl, 63);
    }

    __device__ __forceinline__ int given_len(const PagedShape &sh, int b) const { return span == 1 ? __builtin_amdgcn_readlane(given, b) : given_of(sh, b); }

    __device__ __forceinline__ unsigned int quota(int streams, const PagedSplit &sp) const
    {
        const unsigned int n = total * (unsigned int)streams;
        return max((n + (1u << sp.shift) - 1u) >> sp.shift, sp.least);
    }

    // units of one stream before row b
    __device__ __forceinline__ unsigned int before(const PagedShape &sh, int b, int lane) const
    {
        const int l = b / span;
        unsigned int p = (unsigned int)__builtin_amdgcn_readlane((int)(incl - mine), l);
        if (span > 1) {
            const int r = l * span + lane;
            const unsigned int u = lane < span && r < b ? units(row_len(sh, min(r, sh.B - 1))) : 0u;
            p += (unsigned int)__builtin_amdgcn_readlane((int)wave_scan(u), 63);
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
            const unsigned int in = wave_scan(u);
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
    int fresh;                                           // the position being decoded, -1: none (it is past T_max)
    __device__ __forceinline__ void enter(const PagedShape &sh, const Deal<U> &deal)
    {
        const int given = deal.given_len(sh, b);
        len = taken_len(sh, given);
        fresh = given <= sh.T_max ? len - 1 : -1;
        n_row = Deal<U>::units(len);
    }
    __device__ __forceinline__ bool begin(const PagedShape &sh, const Deal<U> &deal, unsigned int worker, int streams, const PagedSplit &sp, int lane)
    {
        const unsigned int quota = deal.quota(streams, sp), n = deal.total * (unsigned int)streams;
        if (worker >= (1u << sp.shift) || (unsigned long long)worker * quota >= n) return false;
        x = x0 = worker * quota;
        x1 = min(x0 + quota, n);
        b = deal.row_at(sh, (__umulhi(x, sp.by_streams.mul) + x) >> sp.by_streams.shift, lane, &first);
        enter(sh, deal);
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
                ++b;                                     // (units are left, so a row is)
                enter(sh, deal);
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
__device__ __forceinline__ int table_entry(const PagedShape &sh, const int32_t *table, unsigned int u, int lane)
{
    const int row = (int)(u * Tile<DT>::BATCH) + (lane & 7) * Tile<DT>::RPW;
    return table[min(block_of(sh, min(row, sh.T_max - 1)), sh.max_blocks - 1)];
}
// the entry if the lane's load of unit u is one of a row's (u < ue, the row is not over), -1 else
template <int DT>
__device__ __forceinline__ int in_row(const PagedShape &sh, int entry, unsigned int u, unsigned int ue, int len, int lane)
{
    const int row = (int)(u * Tile<DT>::BATCH) + (lane & 7) * Tile<DT>::RPW;
    return u < ue && row < len && (unsigned int)entry < (unsigned int)sh.n_pages ? entry : -1;
}
template <int DT>
__device__ __forceinline__ int look_up(const PagedShape &sh, const int32_t *table, unsigned int u, unsigned int ue, int len, int lane)
{
    return in_row<DT>(sh, table_entry<DT>(sh, table, u, lane), u, ue, len, lane);
}

// the first row of the lane's load among the pool's rows (0 where there is none)
template <int DT>
__device__ __forceinline__ unsigned int pool_row(const PagedShape &sh, int at, unsigned int u, int streams, int s, int lane)
{
    const int row = (int)(u * Tile<DT>::BATCH) + (lane & 7) * Tile<DT>::RPW;
    return at < 0 ? 0u : (unsigned int)(at * streams + s) * (unsigned int)sh.page + (unsigned int)(row - block_of(sh, row) * sh.page);
}

// ONCE: nobody else reads these rows
template <int DT, bool ONCE = true>
__device__ __forceinline__ void request(u32x4 (&buf)[kUnroll], const char *rows, unsigned int row, unsigned int lane_off)
{
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        unsigned long long base = (unsigned long long)rows + (unsigned long long)(unsigned int)__builtin_amdgcn_readlane((int)row, i) * Tile<DT>::ROW_BYTES;
        asm("" : "+s"(base));                // a scalar base and the lanes' offset (else 64-bit additions per lane, and their registers)
        const auto *p = reinterpret_cast<const u32x4 __attribute__((address_space(1))) *>(reinterpret_cast<const char __attribute__((address_space(1))) *>(base) + lane_off);
        buf[i] = ONCE ? __builtin_nontemporal_load(p) : *p;
    }
    asm volatile("" ::: "memory");           // asked for here and not where they are used, one unit later
}

// The query as a lane multiplies it: fp32, beside codes (QB) bf16 pairs.  A code is exact in bf16, and two products of such pairs are added
// to an fp32 sum in one instruction: 16 instructions for sixteen codes where widening to fp32 takes 24, and half the registers.
template <int DT, bool QB>
struct Query {
    float f[Tile<DT>::EPL];
};
template <>
struct Query<DT_E4M3, true> {
    u32x4 pairs[2];
};
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// scores of a unit: lane cg < 8 of a lane group gets that of load cg, row rg + cg * RPW of the unit
template <int DT, bool QB>
__device__ __forceinline__ float dots(const u32x4 (&kb)[kUnroll], const Query<DT, QB> &q, int cg)
{
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        u32x4 raw = kb[i];
        if (DT == DT_E4M3) asm("" : "+v"(raw), "+v"(mine));      // one row is widened at a time (all at once they take 130 registers)
        float dot = 0.f;
        if constexpr (QB) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned int w = raw[e / 2];
                const bf16x2 codes = e % 2 == 0 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
                dot = __builtin_amdgcn_fdot2_f32_bf16(codes, __builtin_bit_cast(bf16x2, (unsigned int)q.pairs[e / 4][e % 4]), dot, false);
            }
        } else {
            float f[Tile<DT>::EPL];
            unpack(raw, f);
#pragma unroll
            for (int e = 0; e < Tile<DT>::EPL; ++e) dot = fmaf(q.f[e], f[e], dot);
        }
        dot = row_sum<DT>(dot);
        mine = cg == i ? dot : mine;
    }
    return mine;
}

// acc += weight * row over a unit's rows; `weight` lies with the lane that owns the row (as in dots), `there` says whether it counts: rows
// that are not attended to and those whose score is -inf do not, else a weight of 0 times an infinite value would be NaN
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
        u32x4 raw = vb[i];
        if (DT == DT_E4M3) asm("" : "+v"(raw), "+v"(acc[0]));
        float f[Tile<DT>::EPL];
        unpack(raw, f);
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

template <int DT, bool QB>
__device__ __forceinline__ void load_query(const char *q, size_t row, int cg, Query<DT, QB> &x)
{
    if constexpr (QB) {
        const u32x4 *p = reinterpret_cast<const u32x4 *>(q + row * (size_t)(kHeadDim * 2) + cg * 32);
        x.pairs[0] = p[0];
        x.pairs[1] = p[1];
    } else {
        load_query<DT>(q, row, cg, CHAI_F32, x.f);           // (q has the type of the rows, or is fp32 beside codes)
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

// ---------------------------------------------------------------------------------------------------------
// The row of the token being decoded, taken from k_new / v_new in the place of what the cache holds there.  A lane has the sixteen bytes
// of the row that it would have loaded, quantised as the append does (the eight lanes of a row of codes together).
// ---------------------------------------------------------------------------------------------------------
template <int DT>
struct FreshRow {
    u32x4 raw;
    float scale;
    __device__ __forceinline__ FreshRow(const char *rows, size_t row, int cg, int q_dtype)
    {
        scale = 1.f;
        if constexpr (DT == DT_E4M3) {
            float f[16], amax = 0.f;
            load_query<DT>(rows, row, cg, q_dtype, f);
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(f[e]));
            amax = dpp_max<0xB1>(amax);
            amax = dpp_max<0x4E>(amax);
            amax = dpp_max<0x141>(amax);
            const float inv = 448.0f / amax;
            scale = amax == 0.f ? 0.f : amax / 448.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = fminf(fmaxf(f[4 * i + e] * inv, -448.0f), 448.0f);
                raw[i] = amax == 0.f ? 0u : e4m3_codes(y[0], y[1], y[2], y[3]);
            }
        } else {
            raw = *reinterpret_cast<const u32x4 *>(rows + row * Tile<DT>::ROW_BYTES + cg * 16);
        }
    }
    // to row `at` of the pool, by one lane group
    __device__ __forceinline__ void store(const char *rows, const float *scales, unsigned int at, int cg) const
    {
        *reinterpret_cast<u32x4 *>(const_cast<char *>(rows) + (size_t)at * Tile<DT>::ROW_BYTES + cg * 16) = raw;
        if (DT == DT_E4M3 && cg == 0) const_cast<float *>(scales)[at] = scale;
    }
};

// Row `local` of a unit whose loads are in buf and begin at rows `row` of the pool becomes the fresh one.
template <int DT>
__device__ __forceinline__ void take_fresh(const FreshRow<DT> &fresh, u32x4 (&buf)[kUnroll], float &row_scale, const char *rows, const float *scales, int at, unsigned int row,
                                           int local, bool keep, int cg, int rg)
{
    const int load = local / Tile<DT>::RPW, group = local % Tile<DT>::RPW;
    if (__builtin_amdgcn_readlane(at, load) < 0) return;     // in no page
    const unsigned int to = (unsigned int)__builtin_amdgcn_readlane((int)row, load) + (unsigned int)group;
    // (selections: an element chosen at run time would put the buffer into memory)
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const bool here = i == load && rg == group;
#pragma unroll
        for (int e = 0; e < 4; ++e) buf[i][e] = here ? fresh.raw[e] : buf[i][e];
        asm("" : "+v"(buf[i]));
    }
    if (DT == DT_E4M3 && cg == load && rg == group) row_scale = fresh.scale;
    if (keep && rg == group) fresh.store(rows, scales, to, cg);
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
// One wave's share of a stream: units ua, ua + step, .. below ue of head h of row b, as weighted mean acc (all lane groups have it), the
// reference m and the sum of exponentials l.  entry0, entry1: table entries of the first two units.  The key of the token being decoded
// goes to slot c if it is the head's own (IDENT).
template <int DT, bool QB, bool IDENT, bool APPEND>
__device__ __forceinline__ void attend_units(const PagedShape &sh, const PagedPages &pg, const char *__restrict__ q, const int32_t *__restrict__ table,
                                             float scale, const char *__restrict__ k_new, const char *__restrict__ v_new, int b, int h, int c, int r, int len,
                                             int fresh, int entry0, int entry1, unsigned int ua, unsigned int ue, unsigned int step, float *strip, int lane, float (&acc)[Tile<DT>::EPL], float &m, float &l)
{
    using TL = Tile<DT>;
    constexpr int U = TL::BATCH;
    const int cg = lane % TL::LPR, rg = lane / TL::LPR;
    const unsigned int lane_off = rg * TL::ROW_BYTES + cg * 16;
    constexpr int q_dtype = DT == DT_BF16 || QB ? CHAI_BF16 : CHAI_F32;
    Query<DT, QB> qf;
    float l_run, down = 1.f;
    for (;;) {
        unsigned int u0 = ua;
        asm volatile("" : "+s"(u0));         // (what the first unit asks for is not kept for the second time around)
        u32x4 kb[kUnroll], vb[kUnroll];
        float ks = 1.f, vs = 1.f;
        int at = in_row<DT>(sh, entry0, u0, ue, len, lane), at1 = in_row<DT>(sh, entry1, u0 + step, ue, len, lane);
        unsigned int krow = pool_row<DT>(sh, at, u0, sh.k, c, lane), vrow = pool_row<DT>(sh, at, u0, sh.H, h, lane);
        request<DT, IDENT>(kb, pg.k, krow, lane_off);
        load_query<DT, QB>(q, (size_t)b * sh.H + r, cg, qf);
        if (DT == DT_E4M3) ks = pg.k_scales[krow + (at < 0 ? 0 : rg)];
        request<DT>(vb, pg.v, vrow, lane_off);
        if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at < 0 ? 0 : rg)];
#pragma unroll
        for (int e = 0; e < TL::EPL; ++e) acc[e] = 0.f;
        m = -INFINITY;
        l_run = 0.f;
        // The last unit apart: what it would ask for is nobody's, and the barrier after it would wait for that (1 x 32 heads of 1024 bf16 tokens
        // 14.4 -> 13.5 us).  The token being decoded is the row's last, so in none of the others.
        auto take = [&](unsigned int u, auto more) __attribute__((always_inline)) {
            constexpr bool kMore = decltype(more)::value;
            const int at2 = kMore ? look_up<DT>(sh, table, u + 2 * step, ue, len, lane) : -1;
            const bool has_fresh = APPEND && !kMore && fresh >= (int)(u * U) && fresh < (int)((u + 1) * U);
            if (has_fresh) take_fresh<DT>(FreshRow<DT>(k_new, (size_t)b * sh.H + r, cg, q_dtype), kb, ks, pg.k, pg.k_scales, at, krow, fresh - (int)(u * U), IDENT, cg, rg);
            const float mine = dots<DT, QB>(kb, qf, cg);
            const bool there = cg < kUnroll && at >= 0 && (int)(u * U) + cg * TL::RPW + rg < len;
            const float sv = there ? scaled<DT>(mine, scale, ks) : -INFINITY;
            if constexpr (kMore) {
                krow = pool_row<DT>(sh, at1, u + step, sh.k, c, lane);
                request<DT, IDENT>(kb, pg.k, krow, lane_off);
                if (DT == DT_E4M3) ks = pg.k_scales[krow + (at1 < 0 ? 0 : rg)];
            }
            if (__any(sv > m)) {
                const float m_new = fmaxf(m, all_max(sv));
                const float f = __expf(m - m_new);
#pragma unroll
                for (int e = 0; e < TL::EPL; ++e) acc[e] *= f;
                l_run *= f;
                m = m_new;
            }
            const float p = __expf(sv - (m == -INFINITY ? 0.f : m)) * down;
            l_run += p;
            if (has_fresh) take_fresh<DT>(FreshRow<DT>(v_new, (size_t)b * sh.H + h, cg, q_dtype), vb, vs, pg.v, pg.v_scales, at, vrow, fresh - (int)(u * U), true, cg, rg);
            const bool counts = sv != -INFINITY;
            weigh<DT>(acc, vb, DT == DT_E4M3 ? (counts ? p * vs : 0.f) : p, counts, strip, cg, rg);
            if constexpr (kMore) {
                vrow = pool_row<DT>(sh, at1, u + step, sh.H, h, lane);
                request<DT>(vb, pg.v, vrow, lane_off);
                if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at1 < 0 ? 0 : rg)];
            }
            at = at1;
            at1 = at2;
        };
        unsigned int u = u0;
#pragma unroll 1
        for (; u + step < ue; u += step) take(u, std::true_type());
        take(u, std::false_type());
        // lane groups; sums beyond the largest float (the quotient is not) are taken again with smaller weights
        bool large = false;
#pragma unroll
        for (int e = 0; e < TL::EPL; ++e) {
            acc[e] = sum_groups<TL::LPR>(acc[e]);
            large = large || !(fabsf(acc[e]) <= kPagedLarge);
        }
        if (!__any(large) || down != 1.f) break;
        down = kPagedDown;
    }
    l = all_sum(l_run);
#pragma unroll
    for (int e = 0; e < TL::EPL; ++e) acc[e] = l == 0.f ? 0.f : acc[e] / l;
    l /= down;
}

template <int DT, bool QB, bool APPEND>
__global__ __launch_bounds__(kBlock, 3) void paged_attend_kernel(
    PagedShape sh, PagedPages pg, PagedSplit sp, const char *__restrict__ q, float scale, const char *__restrict__ k_new,
    const char *__restrict__ v_new, float *__restrict__ partial, float2 *__restrict__ recs, float *__restrict__ out)
{
    using TL = Tile<DT>;
    __shared__ float strip[kWaves][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned int worker = blockIdx.x * kWaves + w;
    const Deal<TL::BATCH> deal(sh, lane);
    Walk<TL::BATCH> wk;
    if (!wk.begin(sh, deal, worker, sh.H, sp, lane)) return;
    do {
        float acc[TL::EPL], m, l;
        const int32_t *table = sh.table + (size_t)wk.b * sh.max_blocks;
        attend_units<DT, QB, true, APPEND>(sh, pg, q, table, scale, k_new, v_new, wk.b, wk.s, wk.s, wk.s, wk.len, wk.fresh,
                                       table_entry<DT>(sh, table, wk.ua, lane), table_entry<DT>(sh, table, wk.ua + 1, lane), wk.ua, wk.ue, 1u, strip[w], lane, acc, m, l);
        const size_t slot = wk.slot(worker);
        float *o = wk.whole() ? out + ((size_t)wk.b * sh.H + wk.s) * kHeadDim : partial + slot * kHeadDim;
        if (lane < TL::LPR) store_floats(o + lane * TL::EPL, acc);
        if (lane == 0 && !wk.whole()) recs[slot] = make_float2(m, l);
    } while (wk.next(sh, deal, sh.H));
}

// The head that workgroup i of a row takes.  Workgroups go round the eight XCDs: the heads, in order of their clusters, are dealt out in
// eight stretches, so that most members of a cluster share the L2 that its keys come through.  (One cluster's heads at a time are counted,
// the scan ends at its own.)
__device__ __forceinline__ int head_by_cluster(const int32_t *__restrict__ h2c, int H, int k, int i, int lane)
{
    const int r = i & 7;
    int p = r * (H >> 3) + min(r, H & 7) + (i >> 3);
    const int c0 = lane < H ? min(max(h2c[min(lane, H - 1)], 0), k - 1) : -1, c1 = lane + 64 < H ? min(max(h2c[min(lane + 64, H - 1)], 0), k - 1) : -1;
    for (int j = 0; j < k; ++j) {
        const unsigned long long m0 = __ballot(c0 == j), m1 = __ballot(c1 == j);
        const int n0 = __popcll(m0), n = n0 + __popcll(m1);
        if (p < n) {
            const bool upper = p >= n0;
            const unsigned long long m = upper ? m1 : m0;
            const int before = __builtin_amdgcn_mbcnt_hi((unsigned int)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned int)m, 0u));
            return __ffsll((long long)(__ballot(before == (upper ? p - n0 : p)) & m)) - 1 + (upper ? 64 : 0);
        }
        p -= n;
    }
    return i;                                // (every head is in a cluster: not reached)
}

// The row that workgroups y * H .. take: of up to 64 rows the y-th in an order of their lengths (`ordered`: rows whose workgroups are the
// first of a CU each).  A CU's loads bound what its workgroups share: the shortest of the first rows come first, and so are on the CUs that
// get a second workgroup of the longest of the others.
__device__ __forceinline__ int row_by_length(const PagedShape &sh, int ordered, int y, int lane)
{
    const int len = taken_len(sh, sh.lens[min(lane, sh.B - 1)]);
    const int key = lane < sh.B ? len * 64 + 63 - lane : -1;             // (lengths are at most 2^24; no two are alike)
    int rank = 0;
    for (int i = 0; i < sh.B; ++i) rank += __builtin_amdgcn_readlane(key, i) > key ? 1 : 0;
    const int want = y < ordered ? ordered - 1 - y : y;
    return __ffsll((long long)__ballot(lane < sh.B && rank == want)) - 1;
}

// Short rows: a workgroup of kRowWaves waves per (head, row), no parts and one launch.  The members of a cluster then each read its keys
// (out of L2), and head h writes the new token's key to every slot that it represents.  Waves take units in turn, each with a softmax of its
// own, and join them in LDS.
// Bound by HBM where the rows fill the CUs evenly: 16 x 32 heads in 8 clusters of up to 2048 bf16 tokens 34.0 us a step, 179 MB at 5.3 TB/s (a
// cluster's keys come from beyond the L2s 1.6 times: 201 MB), 8 x 52 dense of up to 1777 35.6 us, 6.0 TB/s; of codes 23.5 us,
// 3.9 TB/s, of which the products are 5.  Below some 15 us by launch, look-ups one after the other (map and lengths, page, rows) and the longest row:
// 4 x 72 of up to 577 12.5 us, a row of 32 fp32 heads at 256 8.1 us.
template <int DT, bool QB, bool IDENT, bool APPEND, int kRowWaves>
__global__ __launch_bounds__(kRowWaves * 64, kRowWaves == 8 ? 2 : 3) void paged_rows_kernel(PagedShape sh, PagedPages pg, const char *__restrict__ q,
                                                                    const int32_t *__restrict__ h2c, const int32_t *__restrict__ rep, int by_cluster, int ordered, float scale,
                                                                    const char *__restrict__ k_new, const char *__restrict__ v_new, float *__restrict__ out)
{
    using TL = Tile<DT>;
    constexpr unsigned int U = TL::BATCH;
    __shared__ float strip[kRowWaves][64];
    __shared__ float acc_lds[kRowWaves][kHeadDim];
    __shared__ float2 rec_lds[kRowWaves];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = ordered < 0 ? (int)blockIdx.y : row_by_length(sh, ordered, (int)blockIdx.y, lane);
    const int reps = IDENT ? 0 : rep[(size_t)b * sh.k + min(lane, sh.k - 1)];        // (asked for before the cluster is known)
    const int h = IDENT || !by_cluster ? (int)blockIdx.x : head_by_cluster(h2c + (size_t)b * sh.H, sh.H, sh.k, (int)blockIdx.x, lane);
    const int cg = lane % TL::LPR, rg = lane / TL::LPR;
    const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
    const int entry0 = table_entry<DT>(sh, table, (unsigned int)w, lane), entry1 = table_entry<DT>(sh, table, (unsigned int)(w + kRowWaves), lane);
    const int c = IDENT ? h : min(max(h2c[(size_t)b * sh.H + h], 0), sh.k - 1);
    const int r = IDENT ? h : min(max(sh.k <= 64 ? __builtin_amdgcn_readlane(reps, c) : rep[(size_t)b * sh.k + c], 0), sh.H - 1);
    const int given = sh.lens[b], len = taken_len(sh, given), fresh = given <= sh.T_max ? len - 1 : -1;
    const unsigned int n = (unsigned int)(len + U - 1) / U;
    float acc[TL::EPL], m = -INFINITY, l = 0.f;
    if ((unsigned int)w < n) {
        attend_units<DT, QB, IDENT, APPEND>(sh, pg, q, table, scale, k_new, v_new, b, h, c, r, len, fresh, entry0, entry1, (unsigned int)w, n, (unsigned int)kRowWaves,
                                        strip[w], lane,
                                        acc, m, l);
        if (rg == 0) store_floats(&acc_lds[w][cg * TL::EPL], acc);
    }
    if (lane == 0) rec_lds[w] = make_float2(m, l);
    if (APPEND && !IDENT && fresh >= 0 && w == kRowWaves - 1) {
        const int block = block_of(sh, fresh);
        const int at = table[min(block, sh.max_blocks - 1)];
        for (int j0 = 0; j0 < sh.k; j0 += 64) {
            const int rj = j0 + lane < sh.k ? rep[(size_t)b * sh.k + j0 + lane] : -1;
            unsigned long long left = __ballot(rj >= 0 && min(rj, sh.H - 1) == h);
            if (left == 0ull || (unsigned int)at >= (unsigned int)sh.n_pages) continue;
            const FreshRow<DT> row(k_new, (size_t)b * sh.H + h, cg, DT == DT_BF16 || QB ? CHAI_BF16 : CHAI_F32);
            for (; left != 0ull; left &= left - 1ull) {
                const int j = j0 + __ffsll((long long)left) - 1;
                if (rg == 0) row.store(pg.k, pg.k_scales, (unsigned int)(at * sh.k + j) * (unsigned int)sh.page + (unsigned int)(fresh - block * sh.page), cg);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < kHeadDim) {
        float M = -INFINITY, L = 0.f, sum = 0.f, wt[kRowWaves];
#pragma unroll
        for (int i = 0; i < kRowWaves; ++i) M = fmaxf(M, rec_lds[i].x);
#pragma unroll
        for (int i = 0; i < kRowWaves; ++i) {
            const float2 rc = rec_lds[i];
            wt[i] = rc.x == -INFINITY ? rc.y : rc.y * __expf(rc.x - M);      // (only -inf scores: 0, NaN among them: NaN)
            L += wt[i];
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
        for (int i = 0; i < kRowWaves; ++i)
            if ((unsigned int)i < n) sum = fmaf(wt[i] * inv, acc_lds[i][threadIdx.x], sum);
        out[((size_t)b * sh.H + h) * kHeadDim + threadIdx.x] = sum;
    }
}

// ---------------------------------------------------------------------------------------------------------
// Attention in two passes, for layers with fewer clusters than heads whose rows are shared: the keys of a cluster are read once, not once per
// member.  Both are bound by HBM where rows are long: 4 x 32 heads in 4 clusters of 32768 bf16 tokens 24 us of scores (134 MB fetched, 5.5 TB/s), 165 us of
// values (1.08 GB, 6.5 TB/s) and 5 us that join the parts.  64 x 32 of up to 4096 codes, most of them short and some pages absent, take 12.5, 37 and 5 us:
// 248 MB fetched, 4.7 TB/s in all and 5.3 in the values; the scores (48 MB, 3.8 TB/s) are short stretches of many streams, bound by their look-ups.
// Scores: a wave streams keys of its units, writes s[b][j][t] (-inf where nothing is to be attended to, whole units) and the maximum
// and sum of exponentials of every stretch: `whole` of a stream that it took alone, else `parts` of the wave.
// ---------------------------------------------------------------------------------------------------------
template <int DT, bool QB, bool APPEND>
__global__ __launch_bounds__(kBlock, DT == DT_E4M3 ? (APPEND ? 4 : 5) : 6) void paged_scores_kernel(PagedShape sh, PagedPages pg, PagedSplit sp, const char *__restrict__ q,
                                                                 const int32_t *__restrict__ rep, float scale, int T_pad,
                                                                 const char *__restrict__ k_new, float *__restrict__ scores,
                                                                 float2 *__restrict__ whole, float2 *__restrict__ parts)
{
    using TL = Tile<DT>;
    constexpr int U = TL::BATCH, q_dtype = DT == DT_BF16 || QB ? CHAI_BF16 : CHAI_F32;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned int worker = blockIdx.x * kWaves + w;
    const int cg = lane % TL::LPR, rg = lane / TL::LPR;
    const unsigned int lane_off = rg * TL::ROW_BYTES + cg * 16;

    const Deal<U> deal(sh, lane);
    Walk<U> wk;
    if (!wk.begin(sh, deal, worker, sh.k, sp, lane)) return;
    do {
        const int b = wk.b, j = wk.s, len = wk.len;
        const int rj = rep[(size_t)b * sh.k + j], r = min(max(rj, 0), sh.H - 1);
        const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
        u32x4 kb[kUnroll];
        float ks = 1.f;
        int at = look_up<DT>(sh, table, wk.ua, wk.ue, len, lane), at1 = look_up<DT>(sh, table, wk.ua + 1, wk.ue, len, lane);
        unsigned int krow = pool_row<DT>(sh, at, wk.ua, sh.k, j, lane);
        request<DT>(kb, pg.k, krow, lane_off);
        if (DT == DT_E4M3) ks = pg.k_scales[krow + (at < 0 ? 0 : rg)];
        Query<DT, QB> qf;
        load_query<DT, QB>(q, (size_t)b * sh.H + r, cg, qf);
        float *srow = scores + ((size_t)b * sh.k + j) * T_pad;
        float m_run = -INFINITY, l_run = 0.f;            // of the scores that this lane has seen
        auto take = [&](unsigned int u, auto more) __attribute__((always_inline)) {        // (the last unit asks for none)
            constexpr bool kMore = decltype(more)::value;
            const int at2 = kMore ? look_up<DT>(sh, table, u + 2, wk.ue, len, lane) : -1;
            if (APPEND && !kMore && wk.fresh >= (int)(u * U) && wk.fresh < (int)((u + 1) * U))
                take_fresh<DT>(FreshRow<DT>(k_new, (size_t)b * sh.H + r, cg, q_dtype), kb, ks, pg.k, pg.k_scales, at, krow, wk.fresh - (int)(u * U), rj >= 0, cg, rg);
            const float mine = dots<DT, QB>(kb, qf, cg);
            const int t = (int)(u * U) + cg * TL::RPW + rg;
            const bool there = cg < kUnroll && at >= 0 && t < len;
            const float sv = there ? scaled<DT>(mine, scale, ks) : -INFINITY;
            if constexpr (kMore) {
                krow = pool_row<DT>(sh, at1, u + 1, sh.k, j, lane);
                request<DT>(kb, pg.k, krow, lane_off);
                if (DT == DT_E4M3) ks = pg.k_scales[krow + (at1 < 0 ? 0 : rg)];
            }
            if (cg < kUnroll) srow[t] = sv;
            const float m_new = fmaxf(m_run, sv), ref = m_new == -INFINITY ? 0.f : m_new;
            l_run = l_run * __expf(m_run - ref) + __expf(sv - ref);
            m_run = m_new;
            at = at1;
            at1 = at2;
        };
        unsigned int u = wk.ua;
#pragma unroll 1
        for (; u + 1 < wk.ue; ++u) take(u, std::true_type());
        take(u, std::false_type());
        const float M = all_max(m_run);
        const float L = all_sum(m_run == -INFINITY ? l_run : l_run * __expf(m_run - M));     // (lanes that saw only NaN hold it in l_run)
        if (lane == 0) (wk.whole() ? whole[(size_t)b * sh.k + j] : parts[wk.slot(worker)]) = make_float2(M, L);
    } while (wk.next(sh, deal, sh.k));
}

// Maximum and sum of exponentials over a stream's parts.
__device__ __forceinline__ float2 merge(const float2 *parts, const Takers &tk, int lane)
{
    float m = -INFINITY;
    for (unsigned int i = lane; i < tk.n; i += 64) m = fmaxf(m, parts[tk.slot(i)].x);
    const float M = all_max(m);
    float l = 0.f;
    for (unsigned int i = lane; i < tk.n; i += 64) {
        const float2 rc = parts[tk.slot(i)];
        l += rc.x == -INFINITY ? rc.y : rc.y * __expf(rc.x - M);         // (only -inf scores: 0, NaN among them: NaN)
    }
    return make_float2(M, all_sum(l));
}

// Values: a wave streams the values of its units, each weighed by its cluster's probability exp(s - M) / L.
template <int DT, bool APPEND>
__global__ __launch_bounds__(kBlock, DT == DT_E4M3 ? 4 : 5) void paged_values_kernel(PagedShape sh, PagedPages pg, PagedSplit sp, PagedSplit sp_scores,
                                                                 const int32_t *__restrict__ h2c, int T_pad,
                                                                 const char *__restrict__ v_new, int q_dtype, const float *__restrict__ scores, const float2 *__restrict__ whole,
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
        auto take = [&](unsigned int u, auto more) __attribute__((always_inline)) {
            constexpr bool kMore = decltype(more)::value;
            const int at2 = kMore ? look_up<DT>(sh, table, u + 2, wk.ue, len, lane) : -1;
            const bool there = cg < kUnroll && at >= 0 && (int)(u * U) + cg * TL::RPW + rg < len && sv != -INFINITY;
            const float p = there ? __expf(sv - M) * inv : 0.f;
            if (APPEND && !kMore && wk.fresh >= (int)(u * U) && wk.fresh < (int)((u + 1) * U))
                take_fresh<DT>(FreshRow<DT>(v_new, (size_t)b * sh.H + h, cg, q_dtype), vb, vs, pg.v, pg.v_scales, at, vrow, wk.fresh - (int)(u * U), true, cg, rg);
            weigh<DT>(acc, vb, DT == DT_E4M3 ? (there ? p * vs : 0.f) : p, there, strip[w], cg, rg);
            if constexpr (kMore) {
                vrow = pool_row<DT>(sh, at1, u + 1, sh.H, h, lane);
                request<DT>(vb, pg.v, vrow, lane_off);
                if (DT == DT_E4M3) vs = pg.v_scales[vrow + (at1 < 0 ? 0 : rg)];
                sv = srow[(u + 1) * U];
            }
            at = at1;
            at1 = at2;
        };
        unsigned int u = wk.ua;
#pragma unroll 1
        for (; u + 1 < wk.ue; ++u) take(u, std::true_type());
        take(u, std::false_type());
#pragma unroll
        for (int e = 0; e < TL::EPL; ++e) acc[e] = sum_groups<TL::LPR>(acc[e]);
        float *o = wk.whole() ? out + ((size_t)b * sh.H + h) * kHeadDim : partial + wk.slot(worker) * kHeadDim;
        if (rg == 0) store_floats(o + cg * TL::EPL, acc);
    } while (wk.next(sh, deal, sh.H));
}

// Streams that several waves took, 5 us of launch and look-ups, whatever the sizes.  WEIGHED (one pass): out = mean of their parts, each weighed by its sum of exponentials times
// exp(its reference - the largest); else their sum.  JW waves per (row, head), two columns per lane; streams that one wave took are left
// alone, rows without a position get 0.
template <int U, bool WEIGHED, int JW>
__global__ __launch_bounds__(kBlock) void paged_join_kernel(PagedShape sh, PagedSplit sp, const float *__restrict__ partial,
                                                            const float2 *__restrict__ recs, float *__restrict__ out)
{
    __shared__ float2 sums[kWaves][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x * (kWaves / JW) + w / JW, b = blockIdx.y, jw = w % JW;
    if (h >= sh.H) return;                               // (with JW = kWaves none)
    float2 *o = reinterpret_cast<float2 *>(out + ((size_t)b * sh.H + h) * kHeadDim) + lane;
    const Deal<U> deal(sh, lane);
    const unsigned int n_row = Deal<U>::units(taken_len(sh, deal.given_len(sh, b)));
    if (n_row == 0u) {
        if (jw == 0) *o = make_float2(0.f, 0.f);
        return;
    }
    const Takers tk(deal.before(sh, b, lane) * (unsigned int)sh.H + (unsigned int)h * n_row, n_row, deal.quota(sh.H, sp));
    if (tk.n == 1) return;
    float2 sum = make_float2(0.f, 0.f);
    // the first parts are asked for before their weights are known
    const unsigned int per = (tk.n + JW - 1) / JW, i_begin = min((unsigned int)jw * per, tk.n), i_end = min(i_begin + per, tk.n);
    auto part = [&](unsigned int i) { return reinterpret_cast<const float2 *>(partial + tk.slot(min(i, tk.n - 1)) * kHeadDim)[lane]; };
    float2 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = part(i_begin + j);
    float2 st = make_float2(0.f, 1.f);
    if (WEIGHED) st = merge(recs, tk, lane);
    const float inv = st.y == 0.f ? 0.f : 1.f / st.y;
    for (unsigned int i = i_begin; i < i_end; i += 8) {
        float wt = 1.f;
        if (WEIGHED) {
            const float2 rc = recs[tk.slot(min(i + (lane & 7), tk.n - 1))];
            wt = (rc.x == -INFINITY ? rc.y : rc.y * __expf(rc.x - st.x)) * inv;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float wj = WEIGHED ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), j)) : 1.f;
            if (i + j < i_end) {
                sum.x = fmaf(wj, v[j].x, sum.x);
                sum.y = fmaf(wj, v[j].y, sum.y);
            }
            v[j] = part(i + 8 + j);
        }
    }
    if (JW > 1) {
        sums[w][lane] = sum;
        __syncthreads();
        if (jw != 0) return;
#pragma unroll
        for (int i = 1; i < JW; ++i) {
            sum.x += sums[w + i][lane].x;
            sum.y += sums[w + i][lane].y;
        }
    }
    *o = sum;
}

// ---------------------------------------------------------------------------------------------------------
// New rows into pages, and pages into contiguous rows.  A workgroup takes `rows` rows of one request: 1 << shift consecutive tokens (so
// that one new token of many streams fills a workgroup as well) of rows >> shift streams; streams are the k key slots, then the H value
// heads.  Sixteen lanes per row, eight elements each, all rows requested at once.
// Bound by HBM at the rate of a copy: 16 x 40 streams of up to 2043 bf16 tokens quantised 48 us (270 MB, 5.6 TB/s), up to 2048 codes read back 51.5 us
// (5.2 TB/s), 4 x 88 of 512 copied 16 us (92 MB, 5.8 TB/s); one token of 16 x 40 streams 4.0 us, a launch and two look-ups.
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
    const int first = start[b], n = count != nullptr ? min(max(count[b], 0), Tn) : Tn;
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

// where position first + token of a row lies in a pool of `streams` streams (kNowhere beyond n tokens)
__device__ __forceinline__ unsigned int place_of(const PagedShape &sh, const int32_t *table, int first, int token, int n, int streams, int s)
{
    const int pos = (int)((unsigned int)first + (unsigned int)token), block = block_of(sh, max(pos, 0));
    const int at = table[min(block, sh.max_blocks - 1)];
    return token < n && pos >= 0 && block < sh.max_blocks && (unsigned int)at < (unsigned int)sh.n_pages
               ? (unsigned int)(at * streams + s) * (unsigned int)sh.page + (unsigned int)(pos - block * sh.page) : kNowhere;
}

// Row i of every lane group to row at[i] of its pool.
template <int DT, bool BF16>
__device__ __forceinline__ void put_rows(const RawPiece<BF16> (&p)[kMoveUnroll<BF16>], const unsigned int (&at)[kMoveUnroll<BF16>], const bool (&key)[kMoveUnroll<BF16>],
                                         const PagedPages &pg, int piece)
{
    constexpr int kBytes = BF16 ? 2 : 4, N = kMoveUnroll<BF16>;
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
    put_rows<DT, BF16>(p, at, key, pg, piece);
}

// The same for many rows: every wave takes its share of all rows' units, 4 * N tokens of one stream each, whatever the rows' lengths are.
// (A unit's rows asked for before the ones before are stored take twice the registers and, with that, longer.)
template <int DT, bool BF16>
__global__ __launch_bounds__(kBlock, DT == DT_E4M3 ? (BF16 ? 4 : 6) : 7) void paged_append_stream_kernel(PagedShape sh, PagedPages pg, PagedSplit sp, const char *__restrict__ k_new,
                                                                        const char *__restrict__ v_new, long long k_stride, long long v_stride,
                                                                        const int32_t *__restrict__ rep, const int32_t *__restrict__ start)
{
    constexpr int kBytes = BF16 ? 2 : 4, N = kMoveUnroll<BF16>, U = 4 * N;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), piece = lane & 15, rg = lane >> 4;
    const Deal<U> deal(sh, lane);
    Walk<U> wk;
    if (!wk.begin(sh, deal, blockIdx.x * kWaves + w, sh.k + sh.H, sp, lane)) return;
    do {
        const bool key = wk.s < sh.k;
        const int s = key ? wk.s : wk.s - sh.k, streams = key ? sh.k : sh.H, b = wk.b, len = wk.len;
        const int h = key && rep != nullptr ? min(rep[(size_t)b * sh.k + s], sh.H - 1) : s;
        if (h < 0) continue;                 // a slot without a cluster keeps what it holds
        const char *from = (key ? k_new : v_new) + ((size_t)b * sh.H + h) * (key ? k_stride : v_stride) * kBytes;
        const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
        const int first = start[b];
        struct Unit {
            unsigned int at;                 // of row `lane` of the unit
            RawPiece<BF16> p[N];
        };
        auto request = [&](Unit &x, unsigned int u) {
            x.at = place_of(sh, table, first, (int)(u * U) + lane, lane < U && u < wk.ue ? len : 0, streams, s);
#pragma unroll
            for (int i = 0; i < N; ++i) x.p[i].load(from + (size_t)min((int)(u * U) + i * 4 + rg, len - 1) * (kHeadDim * kBytes), piece);
            asm volatile("" ::: "memory");
        };
        auto put = [&](const Unit &x) {
            unsigned int at[N];
            bool keys[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                at[i] = (unsigned int)__shfl((int)x.at, i * 4 + rg);
                keys[i] = key;
            }
            put_rows<DT, BF16>(x.p, at, keys, pg, piece);
        };
        Unit x;
        for (unsigned int u = wk.ua; u < wk.ue; ++u) {
            request(x, u);
            put(x);
        }
    } while (wk.next(sh, deal, sh.k + sh.H));
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

template <int DT, bool BF16>
__global__ __launch_bounds__(kBlock, 8) void paged_gather_stream_kernel(PagedShape sh, PagedPages pg, PagedSplit sp, const int32_t *__restrict__ start,
                                                                        char *__restrict__ k_out, char *__restrict__ v_out)
{
    constexpr int kBytes = BF16 ? 2 : 4, N = kMoveUnroll<BF16>, U = 4 * N;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), piece = lane & 15, rg = lane >> 4;
    const Deal<U> deal(sh, lane);
    Walk<U> wk;
    if (!wk.begin(sh, deal, blockIdx.x * kWaves + w, sh.k + sh.H, sp, lane)) return;
    do {
        const bool key = wk.s < sh.k;
        const int s = key ? wk.s : wk.s - sh.k, streams = key ? sh.k : sh.H, b = wk.b, len = wk.len;
        const char *rows = key ? pg.k : pg.v;
        const float *scales = key ? pg.k_scales : pg.v_scales;
        char *to = (key ? k_out : v_out) + ((size_t)b * streams + s) * sh.T_max * (kHeadDim * kBytes);
        const int32_t *table = sh.table + (size_t)b * sh.max_blocks;
        const int first = start[b];
        auto look = [&](unsigned int u) { return place_of(sh, table, first, (int)(u * U) + lane, lane < U && u < wk.ue ? len : 0, streams, s); };
        struct Unit {
            unsigned int at;                 // of row `lane` of the unit
            float scale;
            RawPiece<BF16> p[N];
            u32x2 codes[N];
        };
        auto request = [&](Unit &x, unsigned int at) {
            x.at = at;
            if (DT == DT_E4M3) x.scale = scales[at != kNowhere ? at : 0u];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const unsigned int r = (unsigned int)__shfl((int)at, i * 4 + rg);
                const size_t row = r != kNowhere ? r : 0u;
                if constexpr (DT == DT_E4M3) x.codes[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(rows) + row * 16 + piece);
                else x.p[i].load(rows + row * (kHeadDim * kBytes), piece);
            }
            asm volatile("" ::: "memory");
        };
        auto put = [&](Unit &x, unsigned int u) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int token = (int)(u * U) + i * 4 + rg;
                if constexpr (DT == DT_E4M3) {
                    const float scale = __shfl(x.scale, i * 4 + rg);
                    float f[8];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x.codes[i][e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x.codes[i][e], true);
                        f[4 * e] = lo.x * scale;
                        f[4 * e + 1] = lo.y * scale;
                        f[4 * e + 2] = hi.x * scale;
                        f[4 * e + 3] = hi.y * scale;
                    }
                    x.p[i].set(f);
                }
                const bool there = (unsigned int)__shfl((int)x.at, i * 4 + rg) != kNowhere;
#pragma unroll
                for (auto &y : x.p[i].x) y = there ? y : u32x4{0u, 0u, 0u, 0u};
                if (token < len) x.p[i].store(to + (size_t)token * (kHeadDim * kBytes), piece);
            }
        };
        Unit x;
        unsigned int next = look(wk.ua);
        for (unsigned int u = wk.ua; u < wk.ue; ++u) {
            const unsigned int at = next;
            next = look(u + 1);
            request(x, at);
            put(x, u);
        }
    } while (wk.next(sh, deal, sh.k + sh.H));
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

// Waves of a launch, a power of two: with 2048 times differ by 3 % (one pass, which has keys and values in flight: between 1024 and 4096).
constexpr unsigned int kStreamWorkers = 4096, kAttendWorkers = 2048, kPagedWorkers = 4096;
// Most waves of one stream: of dense attention and of values, whose parts are joined (1 x 52 dense heads of 8192 bf16 tokens 42.2 us, 43.5
// with 64; 1 x 32 of 2048 15.5, 16.6 with 16), and of scores, of whose parts only two numbers are read again (4 x 4 streams of 32768 bf16
// tokens and their values 212 us with 32, 197 with 64 or 128; 1 x 8 streams 84.9, 72.2 and 66.4).
constexpr unsigned int kPagedParts = 32, kScoreParts = 128;
// The parts of a head are joined by four waves, those of many heads by one each (64 x 32 heads 69.1 / 67.6 us in all, 1 x 52 25.7 / 27.7).
constexpr long long kJoinedByOne = 512;

// Whether a workgroup takes a whole head's row (one launch) or shares of all rows' units go to independent waves (two or three).  The rule goes by
// the longest row, the others' lengths are not known here.  Rows / shares around its limits, in us, the new token's rows written too, bf16 unless
// said, rows of the stated tokens unless spread evenly "to" them:
// * few heads, whose rows a CU's rate bounds: 1 x 32 in 8 clusters of 1024 13.5 / 15.9, 1400 16.0 / 15.8, 2048 21.6 / 15.6; 4 x 32 of 2048 24.1 / 24.5;
// * more heads: 4 x 72 in 16 to 2048 28.1 / 29.8; 16 x 32 in 8 to 2048 34.1 / 41.1, 2048 57.4 / 62.2, to 4000 codes 38.6 / 43.7; 32 x 32 of 2048 111.7 / 111.1;
//   dense 8 x 52 of 2048 68.1 / 72.9, 16 x 32 to 2048 46.0 / 51.0;
// * clustered, beyond 1024: 64 x 32 to 1024 codes 47.1 / 45.6, bf16 67.0 / 67.2.
// It loses where few rows are long, the more so the longer they may be (lengths as the fourth power: 16 x 32 to 2048 26.1 / 24.3, to 4096 codes
// 35.1 / 26.8, with rows of 1 MB 45.2 / 36.3), and where most CUs have one workgroup of long rows and some two (4 x 72 of 2048 46.7 / 39.5, dense 60.0 / 52.6).
static bool take_rows(int B, int H, int T_max, int cache, bool dense)
{
    const long long heads = (long long)B * H, bytes = (long long)T_max * kHeadDim * (cache == CHAI_F32 ? 4 : (cache == CHAI_BF16 ? 2 : 1));
    return bytes <= (heads <= 64 ? 320 : heads <= 128 ? 400 : dense || heads <= 1024 ? 512 : 160) * 1024ll;
}
// Eight waves per row where half the CUs have one, else four (1 x 32 of 1024 bf16 tokens 14.4 against 15.4 us, 4 x 32 15.8 / 16.5, 6 x 32 18.4 /
// 18.0, 16 x 32 38.9 / 32.0).
constexpr long long kFewHeads = 128;
// Heads in order of their clusters from 129 (head, row) pairs on: 16 x 32 in 8 of 577 bf16 tokens 24.4 -> 21.5 us, 1024 38.8 -> 31.8, of 2048 codes
// 43.3 -> 37.3, 4 x 72 in 16 of 1024 30.4 -> 27.2; a row alone pays for the counting (1 x 32 of 1024 14.5 -> 15.0), clusters of less than two
// heads would have nothing for it.  A lane counts two heads at most.
constexpr int kOrderedHeads = 128;
// Rows in order of their lengths where CUs get a second workgroup and not many more (64 x 32 to 1024 codes 47.9 -> 52.6): 16 x 32 to 1024 bf16 tokens
// 23.8 -> 20.8 us, to 2048 42.3 -> 34.1 and of codes 27.9 -> 24.3, 8 x 52 dense to 1024 26.3 -> 22.9; in order of falling lengths throughout 23.1,
// 39.2, 25.9 and 24.9.  Rows that are all alike pay for the look at them: 16 x 32 of 1024 31.9 -> 32.4, 2048 56.9 -> 57.5.
constexpr int kOrderedRows = 64, kCus = 256;
constexpr long long kMostOrdered = 1024;

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

// floor(n / d) = (mulhi(n, mul) + n) >> shift for every 0 <= n < 2^31
static Quotient quotient_by(int d)
{
    Quotient q = {0u, 0};
    while ((1ll << q.shift) < d) ++q.shift;
    q.mul = (unsigned int)((((1ull << q.shift) - (unsigned long long)d) << 32) / (unsigned long long)d + 1ull);
    return q;
}

static PagedSplit make_split(long long units, int streams, unsigned int most, unsigned int least)
{
    PagedSplit sp = {0, least, quotient_by(streams)};
    while ((1ll << sp.shift) < units && (1u << sp.shift) < most) ++sp.shift;
    return sp;
}

static PagedSplit make_paged_split(int B, int streams, int T_max, int cache_dtype, unsigned int workers, unsigned int parts)
{
    const int u = unit_rows(cache_dtype);
    const long long row_units = ((long long)T_max + u - 1) / u;
    return make_split(row_units * B * streams, streams, workers, (unsigned int)((row_units + parts - 1) / parts));
}

// Whether rows are moved by workgroups, a block of tokens each up to the longest row's, or by waves that are dealt units of what there is.
// Workgroups / waves, in us: 16 x 40 streams of 256 tokens quantised 14.6 / 15.9, 512 25.6 / 26.3, 1024 44.8 / 47, evenly up to 1024 35.2 /
// 27.6 and up to 2043 61.5 / 50; read back 12.1 / 13.6, 26.3 / 25.3, 48 / 47, 34.7 / 27.0 and 68 / 52.8; bf16 of 512 copied 33.3 / 32.5, read
// back 32.5 / 31; fp32 70.7 / 79.6 and 97.8 / 70.7.  Many waves of few units each: 4096 to 8192 take up to a tenth longer than 16384 and more.
constexpr long long kStreamedRows = 262144;
constexpr unsigned int kMoveWorkers = 32768;
static bool stream_moves(const PagedShape &sh, int Tn) { return Tn >= 32 && (long long)sh.B * (sh.k + sh.H) * Tn >= kStreamedRows; }

static PagedSplit make_move_split(int B, int streams, int Tn, int dtype)
{
    const int u = 4 * (dtype == CHAI_BF16 ? kMoveUnroll<true> : kMoveUnroll<false>);
    return make_split(((long long)Tn + u - 1) / u * B * streams, streams, kMoveWorkers, 1u);
}

void set_page_division(PagedShape *sh)
{
    const Quotient q = quotient_by(sh->page);
    sh->div_mul = q.mul;
    sh->div_shift = q.shift;
}

template <int DT, bool QB, bool APPEND>
static int paged_attention_typed(const PagedShape &sh, const PagedPages &pg, const char *q, const char *k_new, const char *v_new, int dtype,
                                 const int32_t *h2c, const int32_t *rep, float scale, float *out, char *ws, const PagedPlan &plan, hipStream_t stream)
{
    constexpr int U = Tile<DT>::BATCH, cache = DT;
    float2 *recs = reinterpret_cast<float2 *>(ws + plan.off_recs), *whole = reinterpret_cast<float2 *>(ws + plan.off_whole);
    float *partial = reinterpret_cast<float *>(ws + plan.off_partial), *scores = reinterpret_cast<float *>(ws + plan.off_scores);
    const dim3 block(kBlock);
    auto waves = [](const PagedSplit &sp) { return dim3((workers_of(sp) + kWaves - 1) / kWaves); };
    const KernelEvents none;
    auto join = [&](auto *one, auto *four, const PagedSplit &sp) {
        const bool many = (long long)sh.B * sh.H > kJoinedByOne;
        return (int)launch_kernel(many ? one : four, dim3((unsigned int)(many ? (sh.H + kWaves - 1) / kWaves : sh.H), (unsigned int)sh.B), block, 0, stream, none, sh, sp,
                                  partial, recs, out);
    };
    if (take_rows(sh.B, sh.H, sh.T_max, DT, h2c == nullptr)) {
        const long long heads = (long long)sh.B * sh.H;
        const bool few = heads <= kFewHeads;
        const int ordered = sh.B <= kOrderedRows && heads > kCus && heads <= kMostOrdered ? kCus / sh.H : -1;
        const int by_cluster = !few && sh.H <= kOrderedHeads && 2 * sh.k <= sh.H ? 1 : 0;
        auto rows = [&](auto *kernel) {
            return (int)launch_kernel(kernel, dim3((unsigned int)sh.H, (unsigned int)sh.B), dim3(few ? 512 : 256), 0, stream, none, sh, pg, q, h2c, rep, by_cluster, ordered, scale,
                                      k_new, v_new, out);
        };
        if (h2c == nullptr) return few ? rows(paged_rows_kernel<DT, QB, true, APPEND, 8>) : rows(paged_rows_kernel<DT, QB, true, APPEND, 4>);
        return few ? rows(paged_rows_kernel<DT, QB, false, APPEND, 8>) : rows(paged_rows_kernel<DT, QB, false, APPEND, 4>);
    }
    if (h2c == nullptr) {
        const PagedSplit sp = make_paged_split(sh.B, sh.H, sh.T_max, cache, kAttendWorkers, kPagedParts);
        const hipError_t e = launch_kernel(paged_attend_kernel<DT, QB, APPEND>, waves(sp), block, 0, stream, none, sh, pg, sp, q, scale, k_new, v_new, partial, recs, out);
        if (e != hipSuccess) return (int)e;
        return join(paged_join_kernel<U, true, 1>, paged_join_kernel<U, true, kWaves>, sp);
    }
    const PagedSplit ss = make_paged_split(sh.B, sh.k, sh.T_max, cache, kStreamWorkers, kScoreParts), sv = make_paged_split(sh.B, sh.H, sh.T_max, cache, kStreamWorkers, kPagedParts);
    const int T_pad = padded_tokens(sh.T_max);
    hipError_t e = launch_kernel(paged_scores_kernel<DT, QB, APPEND>, waves(ss), block, 0, stream, none, sh, pg, ss, q, rep, scale, T_pad, k_new, scores, whole, recs);
    if (e != hipSuccess) return (int)e;
    e = launch_kernel(paged_values_kernel<DT, APPEND>, waves(sv), block, 0, stream, none, sh, pg, sv, ss, h2c, T_pad, v_new, dtype, scores, whole, recs, partial, out);
    if (e != hipSuccess) return (int)e;
    return join(paged_join_kernel<U, false, 1>, paged_join_kernel<U, false, kWaves>, sv);
}

int launch_paged_attention(const PagedShape &sh, const PagedPages &pg, const void *q, const void *k_new, const void *v_new, int dtype, int cache_dtype,
                           const int32_t *h2c, const int32_t *rep, float scale, float *out, void *workspace, const PagedPlan &plan, hipStream_t stream)
{
    auto go = [&](auto *typed) {
        return typed(sh, pg, static_cast<const char *>(q), static_cast<const char *>(k_new), static_cast<const char *>(v_new), dtype, h2c, rep, scale, out,
                     static_cast<char *>(workspace), plan, stream);
    };
    if (cache_dtype == CHAI_F32) return k_new ? go(paged_attention_typed<DT_F32, false, true>) : go(paged_attention_typed<DT_F32, false, false>);
    if (cache_dtype == CHAI_BF16) return k_new ? go(paged_attention_typed<DT_BF16, false, true>) : go(paged_attention_typed<DT_BF16, false, false>);
    if (dtype == CHAI_BF16) return k_new ? go(paged_attention_typed<DT_E4M3, true, true>) : go(paged_attention_typed<DT_E4M3, true, false>);
    return k_new ? go(paged_attention_typed<DT_E4M3, false, true>) : go(paged_attention_typed<DT_E4M3, false, false>);
}

int launch_paged_append(const PagedShape &sh, const PagedPages &pg, const void *k_new, const void *v_new, int64_t k_stride,
                        int64_t v_stride, const int32_t *rep, const int32_t *start, const int32_t *count, int Tn, int dtype,
                        int cache_dtype, hipStream_t stream)
{
    if (stream_moves(sh, Tn)) {
        PagedShape each = sh;
        each.lens = count;
        each.T_max = Tn;
        const PagedSplit sp = make_move_split(sh.B, sh.k + sh.H, Tn, dtype);
        auto stream_rows = [&](auto *kernel) {
            return (int)launch_kernel(kernel, dim3((workers_of(sp) + kWaves - 1) / kWaves), dim3(kBlock), 0, stream, KernelEvents(), each, pg, sp,
                                      static_cast<const char *>(k_new), static_cast<const char *>(v_new), k_stride, v_stride, rep, start);
        };
        if (cache_dtype == CHAI_E4M3) return dtype == CHAI_BF16 ? stream_rows(paged_append_stream_kernel<DT_E4M3, true>) : stream_rows(paged_append_stream_kernel<DT_E4M3, false>);
        return dtype == CHAI_BF16 ? stream_rows(paged_append_stream_kernel<DT_BF16, true>) : stream_rows(paged_append_stream_kernel<DT_F32, false>);
    }
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
    if (stream_moves(sh, Tn)) {
        PagedShape each = sh;
        each.lens = count;
        each.T_max = Tn;
        const PagedSplit sp = make_move_split(sh.B, sh.k + sh.H, Tn, dtype);
        auto stream_rows = [&](auto *kernel) {
            return (int)launch_kernel(kernel, dim3((workers_of(sp) + kWaves - 1) / kWaves), dim3(kBlock), 0, stream, KernelEvents(), each, pg, sp, start,
                                      static_cast<char *>(k_out), static_cast<char *>(v_out));
        };
        if (cache_dtype == CHAI_E4M3) return dtype == CHAI_BF16 ? stream_rows(paged_gather_stream_kernel<DT_E4M3, true>) : stream_rows(paged_gather_stream_kernel<DT_E4M3, false>);
        return dtype == CHAI_BF16 ? stream_rows(paged_gather_stream_kernel<DT_BF16, true>) : stream_rows(paged_gather_stream_kernel<DT_F32, false>);
    }
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
