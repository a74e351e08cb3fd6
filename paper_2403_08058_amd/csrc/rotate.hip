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
// 64 turns of every token once, in LDS; then eight lanes take a row, each with 16 elements that are whole pairs (two pieces of 8: at the
// same place of both halves, or any), eight rows of one stream and consecutive tokens a wave.  A thread's first rows are asked for before
// it makes its turns.
#include "chai_rows.h"

#include <hip/hip_ext.h>

namespace chai {

namespace {

constexpr int kTurnTokens = 8;
constexpr int kTurnWaves = kBlock / 64;
constexpr int kTurnUnroll = 4;       // rows of a lane group in flight

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
// dropped without losing the rest: 1 / (2 pi) = hi + lo.
__device__ __forceinline__ double2 turn_of(int pos, double freq)
{
    constexpr double hi = 0x1.45f306dc9c883p-3, lo = -0x1.6b01ec5417056p-57;
    const double p = (double)pos, a = p * freq, a_lo = fma(p, freq, -a);
    const double t = a * hi;
    double rest = fma(a, hi, -t) + fma(a, lo, a_lo * hi);
    const double quarters = rint(4.0 * t);
    rest += fma(-0.25, quarters, t);                     // (exact: both are multiples of the same small power of two)
    double s, c;
    series(rest, s, c);
    const int q = (int)((long long)quarters & 3);        // (an angle below 2^61 quarters: positions are 32 bits, frequencies at most pi)
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
    __device__ __forceinline__ void store(char *row, int p0, int p1) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < kBytes / 16; ++e)
                __builtin_nontemporal_store(x[i * (kBytes / 16) + e], reinterpret_cast<u32x4 *>(row + (i == 0 ? p0 : p1) * kBytes + e * 16));
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

// Pairs of a lane's two pieces: pieces l and l + rot / 16 where they are turned (l < rot / 16), the pieces behind two by two else.
// turns: those of the lane's token, [rot / 2].
template <bool HALVES>
__device__ __forceinline__ void turn(Piece (&p)[2], const double2 *turns, int l, int lanes)
{
    if (l >= lanes) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (HALVES) {
            const double2 t = turns[8 * l + e];
            const double a = p[0].x[e], b = p[1].x[e];
            p[0].x[e] = (float)fma(a, t.x, -(b * t.y));
            p[1].x[e] = (float)fma(a, t.y, b * t.x);
        } else {
            const int i = e >> 2, at = 2 * (e & 3);
            const double2 t = turns[4 * (i == 0 ? l : l + lanes) + (e & 3)];
            const double a = p[i].x[at], b = p[i].x[at + 1];
            p[i].x[at] = (float)fma(a, t.x, -(b * t.y));
            p[i].x[at + 1] = (float)fma(a, t.y, b * t.x);
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

// DT: how keys and values are held; PACKED: into pages, else a block [B,Tn] of a contiguous cache.
template <int DT, bool BF16, bool HALVES, bool PACKED>
__global__ __launch_bounds__(kBlock) void turn_kernel(TurnShape sh, TurnRows rw)
{
    constexpr int kBytes = BF16 ? 2 : 4, kRow = kHeadDim * kBytes;
    __shared__ double2 turns[kTurnTokens][kHeadDim / 2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane & 7;
    const int lanes = sh.rot / 16, p0 = l < lanes ? l : 2 * l, p1 = l < lanes ? l + lanes : 2 * l + 1;
    const int q_streams = rw.q != nullptr ? sh.k : 0, turned = q_streams + (rw.k != nullptr ? sh.k : 0), streams = turned + (PACKED ? sh.H : 0);

    // the lane group's token
    const int n = blockIdx.x * kTurnTokens + (lane >> 3);
    bool there = n < sh.N;
    int b = 0, i = 0, slot = -1;
    if constexpr (PACKED) {
        if (there) {
            b = sh.rows[n];
            slot = sh.slots[n];
        }
        there = there && (unsigned int)b < (unsigned int)sh.B;
        b = there ? b : 0;
    } else {
        b = there ? n / sh.Tn : 0;
        i = n - b * sh.Tn;
    }
    long long place = -1;                                // packed: of a stream's row in its page, and the page
    int at_page = 0;
    if constexpr (PACKED) {
        if (there && slot >= 0) {
            at_page = (int)((__umulhi((unsigned int)slot, sh.div_mul) + (unsigned int)slot) >> sh.div_shift);
            place = at_page < sh.n_pages ? slot - at_page * sh.page : -1;
        }
    }
    const int32_t *rep = sh.rep != nullptr ? sh.rep + (size_t)b * sh.k : nullptr;
    const bool q_in_place = rw.q == rw.q_out;

    struct Row {
        const char *from;
        char *to;                                        // (codes: the number of the row)
        Pair16<BF16> x;
    };
    auto request = [&](Row &r, int s) __attribute__((always_inline)) {
        r.to = nullptr;
        r.from = nullptr;
        if (!there || s >= streams) return;
        if (s >= turned) {                               // values
            const int h = s - turned;
            if (place < 0) return;
            r.from = rw.v + ((long long)n * rw.v_stride + h * kHeadDim) * kBytes;
            const long long to = ((long long)at_page * sh.H + h) * sh.page + place;
            r.to = rw.v_out + to * (DT == DT_E4M3 ? kHeadDim : kRow);
        } else {
            const bool key = s >= q_streams;
            const int j = key ? s - q_streams : s;
            const int h = rep != nullptr ? min(rep[j], sh.H - 1) : j;
            if (h < 0) return;                           // a slot without a cluster
            if (!key) {
                if (q_in_place && rep != nullptr) {      // a head that stands in several slots is turned once
                    for (int o = 0; o < j; ++o)
                        if (min(rep[o], sh.H - 1) == h) return;
                }
                r.from = rw.q + (PACKED ? (long long)n * rw.q_stride + h * kHeadDim : ((long long)b * sh.H + h) * rw.q_stride + (long long)i * kHeadDim) * kBytes;
                r.to = rw.q_out + (PACKED ? (long long)n * sh.H + h : ((long long)b * sh.H + h) * sh.Tn + i) * kRow;
            } else if constexpr (PACKED) {
                if (place < 0) return;
                r.from = rw.k + ((long long)n * rw.k_stride + (sh.by_slot ? j : h) * kHeadDim) * kBytes;
                const long long to = ((long long)at_page * sh.k + j) * sh.page + place;
                r.to = rw.k_out + to * (DT == DT_E4M3 ? kHeadDim : kRow);
            } else {
                r.from = rw.k + (((long long)b * sh.k + j) * rw.k_stride + (long long)i * kHeadDim) * kBytes;
                r.to = rw.k_out + (((long long)b * sh.k + j) * sh.Tc_cap + sh.pos0 + i) * kRow;
            }
        }
        r.x.load(r.from, p0, p1);
    };
    auto finish = [&](Row &r, int s) __attribute__((always_inline)) {
        if (r.to == nullptr) return;
        const bool value = s >= turned, coded = DT == DT_E4M3 && s >= q_streams;
        if (value && !coded) {
            r.x.store(r.to, p0, p1);
            return;
        }
        Piece p[2];
        r.x.widen(p);
        if (!value) turn<HALVES>(p, turns[lane >> 3], l, lanes);
        if (!coded) {
            r.x.set(p);
            r.x.store(r.to, p0, p1);
            return;
        }
        if constexpr (DT == DT_E4M3) {
            const float amax = largest_of_two(p);
            const float inv = amax == 0.f ? 0.f : 448.0f / amax;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<uint2 *>(r.to + (e == 0 ? p0 : p1) * 8) = amax == 0.f ? make_uint2(0u, 0u) : codes_of(p[e], inv);
            if (l == 0) (value ? rw.v_scales + (r.to - rw.v_out) / kHeadDim : rw.k_scales + (r.to - rw.k_out) / kHeadDim)[0] = amax == 0.f ? 0.f : amax / 448.0f;
        }
    };

    const int parts = gridDim.y * kTurnWaves, s0 = blockIdx.y * kTurnWaves + w;
    Row row[kTurnUnroll];
#pragma unroll
    for (int u = 0; u < kTurnUnroll; ++u) request(row[u], s0 + u * parts);
    if ((int)blockIdx.y * kTurnWaves < turned) {         // (a workgroup of values alone needs no turns)
        const int half = sh.rot / 2;
        for (int x = tid; x < kTurnTokens * 64; x += kBlock) {
            const int token = x >> 6, f = x & 63, m = blockIdx.x * kTurnTokens + token;
            if (f < half && m < sh.N) {
                const int pos = sh.positions != nullptr ? sh.positions[m] : sh.pos0 + m % sh.Tn;
                const double2 t = turn_of(pos, sh.freq[f]);
                turns[token][f] = double2{t.x * sh.gain, t.y * sh.gain};
            }
        }
    }
    __syncthreads();
    for (int s = s0; s < streams; s += kTurnUnroll * parts) {
#pragma unroll
        for (int u = 0; u < kTurnUnroll; ++u) finish(row[u], s + u * parts);
        if (s + kTurnUnroll * parts < streams) {
#pragma unroll
            for (int u = 0; u < kTurnUnroll; ++u) request(row[u], s + (kTurnUnroll + u) * parts);
        }
    }
}

// Workgroups of a group of tokens: as many as bring the chip to two per CU, at most one for every four streams.
unsigned int parts_of(long long groups, int streams)
{
    const long long most = (streams + kTurnWaves - 1) / kTurnWaves, want = (512 + groups - 1) / groups;
    return (unsigned int)(want < most ? want : most);
}

template <int DT, bool BF16, bool PACKED>
int launch_turn(const TurnShape &sh, const TurnRows &rows, int layout, int streams, hipStream_t stream)
{
    const long long groups = ((long long)sh.N + kTurnTokens - 1) / kTurnTokens;
    const dim3 grid((unsigned int)groups, parts_of(groups, streams));
    return (int)launch_kernel(layout == CHAI_ROPE_HALVES ? turn_kernel<DT, BF16, true, PACKED> : turn_kernel<DT, BF16, false, PACKED>, grid, dim3(kBlock), 0,
                              stream, KernelEvents{}, sh, rows);
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
