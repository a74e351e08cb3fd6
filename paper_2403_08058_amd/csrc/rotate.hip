// Rotary positions: queries and keys turned by the positions of their tokens, in a contiguous cache or on the way into pages.
//
// The first `rot` elements of a row of 128 are rot / 2 pairs; pair i of a token at position p is turned by the angle p * freq[i]:
//     (a, b) -> gain * (a cos - b sin, a sin + b cos)
// with a, b = elements i and i + rot / 2 (halves), or 2 i and 2 i + 1 (pairs).  The rest of the row stays as it is.
//
// All of it is in 64 bits, rounded once to 32 and from there to the type that is stored.  An angle of a far position needs them (a
// million radians in 32 bits are off by up to 1/32); the products then cost no more than 32-bit ones would (the rates of 64-bit and of
// unpacked 32-bit operations are the same here), and codes of 8 bits, which tell apart what a last bit of 32 decides, are those of the
// exact rows.
//
// A workgroup takes kTurnTokens tokens and a part of their streams (queries of representatives, keys, values).  Its threads make the
// 64 turns of every token once, in LDS, while their first rows are on the way; eight lanes take a row, each with 16 elements that are
// whole pairs: two pieces of 8, at the same place of both halves, or a cache line apart where pairs are neighbours.
//
// What bounds it: HBM, at the rate of a copy.  16 rows x 32 heads in 8 clusters, 2043 positions 50.2 us (5.3 TB/s read + written), 4 x 52
// dense heads, 777 far positions 30.1 (5.5), 4 x 72 dense heads of up to 1000 tokens into pages 52.5 (5.3), 64 rows with 8 prompts into
// pages of codes 36.1 (5.0).  On the way there, in us of these four: four rows of a lane under way 62, 43, 77 and 50; pieces that make up
// whole lines of 128 bytes in each store 62, 31, 57 and 50 (parts of two lines, stored past the caches, are written twice); one row
// under way, and registers for seven waves a SIMD to make up for it, 50.2, 30.1, 54.4 and 38.5.  Five: 52.1 us for the first, eight: 57.
// Workgroups enough to even out the last round: 4096; 2048 take 32 us for the second, 8192 56 for the first, whose turns are made once
// for every part.
#include "chai_rows.h"

#include <hip/hip_ext.h>

namespace chai {

namespace {

constexpr int kTurnTokens = 8;
constexpr int kTurnWaves = kBlock / 64;
constexpr int kTurnGroups = 4096;    // workgroups that a call is cut into at least, if it has so many rows

// sin and cos of a turn of x times 2 pi, |x| <= 1/8: the power series at 2 pi x, to the term below 2^-56
__device__ __forceinline__ void series(double x, double &s, double &c)
{
    const double y = 6.283185307179586476925 * x, z = y * y;
    double a = 1.0 / 355687428096000.0;                  // 1/17!
    a = fma(a, z, -1.0 / 1307674368000.0);
    a = fma(a, z, 1.0 / 6227020800.0);
    a = fma(a, z, -1.0 / 39916800.0);
    a = fma(a, z, 1.0 / 362880.0);
    a = fma(a, z, -1.0 / 5040.0);
    a = fma(a, z, 1.0 / 120.0);
    a = fma(a, z, -1.0 / 6.0);
    s = fma(a * z, y, y);
    double b = 1.0 / 20922789888000.0;                   // 1/16!
    b = fma(b, z, -1.0 / 87178291200.0);
    b = fma(b, z, 1.0 / 479001600.0);
    b = fma(b, z, -1.0 / 3628800.0);
    b = fma(b, z, 1.0 / 40320.0);
    b = fma(b, z, -1.0 / 720.0);
    b = fma(b, z, 1.0 / 24.0);
    b = fma(b, z, -0.5);
    c = fma(b, z, 1.0);
}

// cos and sin of pos * freq.  The product is taken exactly, as a sum of two, and divided by 2 pi to 106 bits, so that whole turns can be
// dropped without losing the rest: 1 / (2 pi) = hi + lo.  (Without contraction: t is the rounded product, whose rest is kept apart.)
__device__ __forceinline__ double2 turn_of(int pos, double freq)
{
#pragma clang fp contract(off)
    constexpr double hi = 0x1.45f306dc9c883p-3, lo = -0x1.6b01ec5417056p-57;
    const double p = (double)pos, a = p * freq, a_lo = fma(p, freq, -a);
    const double t = a * hi;
    double rest = fma(a, hi, -t) + fma(a, lo, a_lo * hi);
    const double r = t - rint(t), quarters = rint(4.0 * r);      // (exact, like the next: all are multiples of t's last place)
    rest += fma(-0.25, quarters, r);
    double s, c;
    series(rest, s, c);
    const int q = (int)quarters & 3;
    const double x = (q & 1) ? s : c, y = (q & 1) ? c : s;
    return double2{q == 1 || q == 2 ? -x : x, q >= 2 ? -y : y};
}

// 16 elements of a row: two pieces of 8
template <bool BF16>
struct Pair16 {
    u32x4 x[BF16 ? 2 : 4];
    static constexpr int kBytes = BF16 ? 16 : 32;        // of a piece
    __device__ __forceinline__ void load(const char *row, int p0, int p1)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < kBytes / 16; ++e) x[i * (kBytes / 16) + e] = stream16(row + (i == 0 ? p0 : p1) * kBytes + e * 16);
    }
    // LINES: what eight lanes store at once are whole cache lines, which nobody has to keep for what is missing of them
    template <bool LINES>
    __device__ __forceinline__ void store(char *row, int p0, int p1) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < kBytes / 16; ++e) {
                u32x4 *to = reinterpret_cast<u32x4 *>(row + (i == 0 ? p0 : p1) * kBytes + e * 16);
                if (LINES) __builtin_nontemporal_store(x[i * (kBytes / 16) + e], to);
                else *to = x[i * (kBytes / 16) + e];
            }
    }
    __device__ __forceinline__ void widen(Piece (&p)[2]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (BF16) {
                unpack(x[i], p[i].x);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) p[i].x[e] = __uint_as_float(x[2 * i + e / 4][e % 4]);
            }
        }
    }
    __device__ __forceinline__ void set(const Piece (&p)[2])
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (BF16) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[i][e] = __builtin_bit_cast(unsigned int, __builtin_convertvector(f32x2{p[i].x[2 * e], p[i].x[2 * e + 1]}, bf16x2));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[2 * i + e / 4][e % 4] = __float_as_uint(p[i].x[e]);
            }
        }
    }
};

// Turns the pairs of a lane's two pieces; turns: those of the lane's token, [rot / 2]; lanes = rot / 16.
template <bool HALVES>
__device__ __forceinline__ void turn(Piece (&p)[2], const double2 *turns, int l, int lanes)
{
    if constexpr (HALVES) {
        if (l >= lanes) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double2 t = turns[8 * l + e];
            const double a = p[0].x[e], b = p[1].x[e];
            p[0].x[e] = (float)fma(a, t.x, -(b * t.y));
            p[1].x[e] = (float)fma(a, t.y, b * t.x);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int piece = l + 8 * i;
            if (piece >= 2 * lanes) continue;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const double2 t = turns[4 * piece + e / 2];
                const double a = p[i].x[e], b = p[i].x[e + 1];
                p[i].x[e] = (float)fma(a, t.x, -(b * t.y));
                p[i].x[e + 1] = (float)fma(a, t.y, b * t.x);
            }
        }
    }
}

// largest magnitude over the eight lanes of a row
__device__ __forceinline__ float largest_of_two(const Piece (&p)[2])
{
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(p[i].x[e]));
    amax = dpp_max<0xB1>(amax);                          // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror
    amax = dpp_max<0x4E>(amax);
    return dpp_max<0x141>(amax);
}

// DT: how keys and values are held; PACKED: into pages, else a block [B,Tn] of a contiguous cache.  A wave's eight rows
// lie side by side: neighbouring streams of one token where tokens are packed (ALONG), else one stream's of neighbouring tokens.
template <int DT, bool BF16, bool HALVES, bool PACKED, bool LINES>
__global__ __launch_bounds__(kBlock, 7) void turn_kernel(TurnShape sh, TurnRows rw, int per)
{
    constexpr bool ALONG = PACKED;
    constexpr int kBytes = BF16 ? 2 : 4, kRow = kHeadDim * kBytes;
    __shared__ double2 turns[kTurnTokens][kHeadDim / 2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane & 7, rg = lane >> 3;
    const int lanes = sh.rot / 16, p0 = !HALVES || l < lanes ? l : l + lanes, p1 = HALVES && l < lanes ? l + lanes : l + 8;
    const int q_streams = rw.q != nullptr ? sh.k : 0, turned = q_streams + (rw.k != nullptr ? sh.k : 0), streams = turned + (PACKED ? sh.H : 0);
    const int n0 = blockIdx.x * kTurnTokens, tokens = min(kTurnTokens, sh.N - n0), across = (streams + 7) / 8;
    // This workgroup's eights of rows: streams, or (token, eight streams), in whose order tokens change first, so that rows of a page are
    // written side by side (4 x 72 heads of up to 1000 tokens 54.5 -> 52.8 us), but last where they are quantised, which takes the time
    // (64 rows with 8 prompts 39.7 -> 37.5).
    constexpr bool kTokensFirst = DT != DT_E4M3;
    const int items = ALONG ? tokens * across : streams, i0 = blockIdx.y * per, i1 = min(i0 + per, items);
    if (i0 >= i1) return;

    // what is known of token n0 + rg: its row, its slot and, of blocks, its number in the row
    const int mine = n0 + rg;
    int row = -1, slot = -1, number = 0;
    if (mine < sh.N) {
        if constexpr (PACKED) {
            row = sh.rows[mine];
            slot = sh.slots[mine];
        } else {
            row = mine / sh.Tn;
            number = mine - row * sh.Tn;
        }
    }
    const bool q_in_place = rw.q == rw.q_out;

    struct Row {
        char *to;                                        // (NULL: none; codes: the row of 128 bytes)
        int t;
        bool turned, coded, value;
        Pair16<BF16> x;
    };
    auto request = [&](Row &r, int item) __attribute__((always_inline)) {
        r.to = nullptr;
        const int t = !ALONG ? rg : kTokensFirst ? item % tokens : item / across, s = !ALONG ? item : (kTokensFirst ? item / tokens : item - t * across) * 8 + rg;
        const int b = ALONG ? __builtin_amdgcn_readlane(row, t * 8) : row, at = ALONG ? __builtin_amdgcn_readlane(slot, t * 8) : slot, n = n0 + t;
        r.t = t;
        r.turned = s < turned;
        r.value = s >= turned;
        r.coded = DT == DT_E4M3 && s >= q_streams;
        if (item >= i1 || s >= streams || (unsigned int)b >= (unsigned int)sh.B) return;
        // packed: the row's place in its stream's pages
        int page = 0;
        bool placed = false;
        if constexpr (PACKED) {
            page = (int)((__umulhi((unsigned int)max(at, 0), sh.div_mul) + (unsigned int)max(at, 0)) >> sh.div_shift);
            placed = at >= 0 && page < sh.n_pages;
        }
        auto in_pages = [&](char *pages, int of, int stream) {
            return pages + (((long long)page * of + stream) * sh.page + (at - page * sh.page)) * (DT == DT_E4M3 ? kHeadDim : kRow);
        };
        const char *from;
        if (s >= turned) {
            if (!placed) return;
            const int h = s - turned;
            from = rw.v + (n * rw.v_stride + h * rw.v_head) * kBytes;
            r.to = in_pages(rw.v_out, sh.H, h);
        } else {
            const bool key = s >= q_streams;
            const int j = key ? s - q_streams : s;
            const int32_t *rep = sh.rep != nullptr ? sh.rep + (long long)b * sh.k : nullptr;
            const int h = rep != nullptr ? min(rep[j], sh.H - 1) : j;
            if (h < 0) return;                           // a slot without a cluster
            if (!key) {
                // A head that stands in several slots is turned once.  (A look at every slot before: 16 x 2043 tokens of 32 heads in 8 clusters
                // 54.6 us in place, 49.2 elsewhere, of 72 in 16 117 and 100, 4 x 777 of 72 with maps of all 88 and 44.)
                if (q_in_place && rep != nullptr) {
                    for (int o = 0; o < j; ++o)
                        if (min(rep[o], sh.H - 1) == h) return;
                }
                from = rw.q + (PACKED ? n * rw.q_stride + h * rw.q_head : ((long long)b * sh.H + h) * rw.q_stride + (long long)number * kHeadDim) * kBytes;
                r.to = rw.q_out + (PACKED ? (n * rw.out_stride + h * rw.out_head) * kBytes : (((long long)b * sh.H + h) * sh.Tn + number) * kRow);
            } else if constexpr (PACKED) {
                if (!placed) return;
                from = rw.k + (n * rw.k_stride + (sh.by_slot ? j : h) * rw.k_head) * kBytes;
                r.to = in_pages(rw.k_out, sh.k, j);
            } else {
                from = rw.k + (((long long)b * sh.k + j) * rw.k_stride + (long long)number * kHeadDim) * kBytes;
                r.to = rw.k_out + (((long long)b * sh.k + j) * sh.Tc_cap + sh.pos0 + number) * kRow;
            }
        }
        r.x.load(from, p0, p1);
    };
    auto finish = [&](Row &r) __attribute__((always_inline)) {
        if (r.to == nullptr) return;
        if (!r.turned && !r.coded) {
            r.x.template store<LINES>(r.to, p0, p1);
            return;
        }
        Piece p[2];
        r.x.widen(p);
        if (r.turned) turn<HALVES>(p, turns[r.t], l, lanes);
        if (!r.coded) {
            r.x.set(p);
            r.x.template store<LINES>(r.to, p0, p1);
            return;
        }
        if constexpr (DT == DT_E4M3) {
            const float amax = largest_of_two(p);
            const float inv = amax == 0.f ? 0.f : 448.0f / amax;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<uint2 *>(r.to + (e == 0 ? p0 : p1) * 8) = amax == 0.f ? make_uint2(0u, 0u) : codes_of(p[e], inv);
            if (l == 0) (r.value ? rw.v_scales + (r.to - rw.v_out) / kHeadDim : rw.k_scales + (r.to - rw.k_out) / kHeadDim)[0] = amax == 0.f ? 0.f : amax / 448.0f;
        }
    };

    Row r;
    request(r, i0 + w);
    // the turns of the tokens that the workgroup has turned rows of
    const int t0 = ALONG && !kTokensFirst ? i0 / across : 0, t1 = ALONG && !kTokensFirst ? (i1 - 1) / across + 1 : tokens, half = sh.rot / 2;
    if (ALONG || i0 < turned) {
        for (int x = t0 * 64 + tid; x < t1 * 64; x += kBlock) {
            const int token = x >> 6, f = x & 63, m = n0 + token;
            if (f < half && m < sh.N) {
                const int pos = sh.positions != nullptr ? sh.positions[m] : sh.pos0 + m % sh.Tn;
                const double2 t = turn_of(pos, sh.freq[f]);
                turns[token][f] = double2{t.x * sh.gain, t.y * sh.gain};
            }
        }
    }
    __syncthreads();
    for (int i = i0 + w; i < i1; i += kTurnWaves) {
        finish(r);
        if (i + kTurnWaves < i1) request(r, i + kTurnWaves);
    }
}

// Workgroups of eight tokens: as many as bring the chip to kTurnGroups, none with less than a row for each of its lane groups.
template <int DT, bool BF16, bool PACKED>
int launch_turn(const TurnShape &sh, const TurnRows &rows, int layout, int streams, hipStream_t stream)
{
    const long long groups = ((long long)sh.N + kTurnTokens - 1) / kTurnTokens;
    const int items = PACKED ? (int)(sh.N < kTurnTokens ? sh.N : kTurnTokens) * ((streams + 7) / 8) : streams;
    const long long most = (items + kTurnWaves - 1) / kTurnWaves, want = groups < kTurnGroups ? kTurnGroups / groups : 1, parts = want < most ? want : most;
    int per = (int)((items + parts - 1) / parts);
    per = (per + kTurnWaves - 1) / kTurnWaves * kTurnWaves;
    const dim3 grid((unsigned int)groups, (unsigned int)((items + per - 1) / per));
    // Whole lines leave the caches at once: rows of bf16, but for halves of a part of the row, whose pieces lie in between (4 x 52 dense
    // heads, 777 positions, 64 of 128 elements 35 us, 41 if those did; fp32 rows of half the positions 45 and 54).
    const bool halves = layout == CHAI_ROPE_HALVES, lines = BF16 && (!halves || sh.rot == 0 || sh.rot == kHeadDim);
    auto *kernel = !halves ? turn_kernel<DT, BF16, false, PACKED, BF16> : lines ? turn_kernel<DT, BF16, true, PACKED, BF16> : turn_kernel<DT, BF16, true, PACKED, false>;
    return (int)launch_kernel(kernel, grid, dim3(kBlock), 0, stream, KernelEvents{}, sh, rows, per);
}

}  // namespace

int launch_rotate(const TurnShape &sh, const TurnRows &rows, int layout, int dtype, hipStream_t stream)
{
    const int streams = (rows.q ? sh.k : 0) + (rows.k ? sh.k : 0);
    return dtype == CHAI_BF16 ? launch_turn<DT_BF16, true, false>(sh, rows, layout, streams, stream)
                              : launch_turn<DT_F32, false, false>(sh, rows, layout, streams, stream);
}

int launch_append_packed(const TurnShape &sh, const TurnRows &rows, int layout, int dtype, int cache_dtype, hipStream_t stream)
{
    const int streams = (rows.q ? sh.k : 0) + sh.k + sh.H;
    if (cache_dtype == CHAI_E4M3)
        return dtype == CHAI_BF16 ? launch_turn<DT_E4M3, true, true>(sh, rows, layout, streams, stream)
                                  : launch_turn<DT_E4M3, false, true>(sh, rows, layout, streams, stream);
    return dtype == CHAI_BF16 ? launch_turn<DT_BF16, true, true>(sh, rows, layout, streams, stream)
                              : launch_turn<DT_F32, false, true>(sh, rows, layout, streams, stream);
}

}  // namespace chai
