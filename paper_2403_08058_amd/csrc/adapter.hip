// The first half of a low-rank adapter: t = s_a x A_a^T of every token, a = the adapter of the token's row.  The projections add the second
// half, t B_a^T, to what they sum up (project.hip).
//
//   x [B,Tn,D], A [n,R,D] bf16, queries' and keys' apart;  t [B,Tn][2][chunks][3][16] bf16: of sixteen ranks the upper 8 bits of t (half
//   of that number, which is taken twice), the next 8 and the last 8: all of its 24.  (In the upper 16 alone it is the largest error of the
//   call before its rounding: it then decides that of 0.17 % of the outputs, 16 rows x 1 token, width 4096, rank 16, and the order of all
//   sums together that of 0.02 %.  The lower 8 cost nothing there; 1 x 1777 tokens of 16 heads, rank 64, 160 -> 164 us, 4 x 2043 of 8, rank
//   128, 181 -> 194.)
//
// A workgroup takes the ranks of U units of 8 (of queries, then of keys) for 8 XT tokens of one row.  As in the projections of few tokens,
// its waves deal the contraction out in blocks of 64 elements and stream their blocks, ranks and tokens, through rings of their own in LDS,
// without a barrier before the sums of all waves are added in wave order.
//
// What bounds it: of prompts HBM, which the activations come from once more (16 rows x 2043 tokens, width 4096: 293 MB fetched in 65 us, 4.5
// TB/s; a stretch of blocks for each wave, so that a row's neighbouring lines are asked for by one, takes a seventh less, but the projections
// that follow run at the clock that their power leaves and give it back, and few tokens take 0.3 to 1 us longer so).  Making t in the
// projections' own tiles instead would cost them an eighth more products.  Of few tokens launch, look-up and ramp, 4 to 5 us; rows of one
// adapter in one workgroup, which reads its ranks once, take 0.8 us more to be found and give nothing back (L2 holds them).
#include "chai_internal.h"

#include <hip/hip_ext.h>

#include <type_traits>
#include <utility>

namespace chai {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

union Frag {
    u32x4 raw;
    bf16x8 bf;
};

template <typename F, int... I>
__device__ __forceinline__ void unroll_seq(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unroll(F &&f)
{
    unroll_seq(f, std::make_integer_sequence<int, N>{});
}

// y = 2 hi + mid + lo, each of 8 bits of mantissa and of y's sign, none 0 unless y is: cut below the number next to it, so that something
// is left for the next.  0, infinities and NaN are all three.  (Below 2^-95 what is left is too small for a bf16, and 0.)
struct Parts {
    float hi, mid, lo;
};
__device__ __forceinline__ Parts parts_of(float y)
{
#pragma clang fp contract(off)
    auto below = [](float x) { return __uint_as_float((__float_as_uint(x) - 1u) & 0xffff0000u); };
    if (y == 0.f || y - y != 0.f) return Parts{y, y, y};
    const float hi = below(y), rest = y - hi, mid = below(rest);
    return Parts{0.5f * hi, mid, rest - mid};
}

constexpr int wave_bytes(int waves) { return waves > 8 ? 10 * 1024 : 20 * 1024; }      // ring of a wave
constexpr int kAdMostAhead = 8;

template <int U, int XT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void adapter_down_kernel(const char *__restrict__ x, const int32_t *__restrict__ ids,
                                                                  const char *__restrict__ a_q, const char *__restrict__ a_k,
                                                                  const float *__restrict__ scales, int n, int R, int Tn, int D, int tiles,
                                                                  int groups, unsigned int items, char *__restrict__ t)
{
    constexpr int NB = (U + 1) / 2, TT = (XT + 1) / 2, kLoads = U + XT, kBytes = kLoads * 1024, kAdWaveBytes = wave_bytes(WAVES);
    constexpr int N = kAdWaveBytes / kBytes < kAdMostAhead ? kAdWaveBytes / kBytes : kAdMostAhead;       // blocks of a ring
    static_assert(N >= 2 && NB * TT * 1024 <= kAdWaveBytes, "a block ahead; the sums fit");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // items: (row, tile of tokens, group of ranks), the groups of a tile, which read the same tokens, on one XCD
    const unsigned int local = blockIdx.x >> 3, item = (local / (unsigned int)groups * 8u + (blockIdx.x & 7u)) * (unsigned int)groups + local % (unsigned int)groups;
    if (item >= items) return;
    const int group = (int)(item % (unsigned int)groups), tile = (int)(item / (unsigned int)groups), b = tile / tiles, c0 = (tile - b * tiles) * 8 * XT;
    const int a = ids[b];
    if ((unsigned int)a >= (unsigned int)n) return;      // (t of these rows is not read)
    const int each = R / 8, first = a_q == nullptr ? each : 0, total = (a_q != nullptr ? each : 0) + (a_k != nullptr ? each : 0);
    const int u0 = group * U;                            // units of the group: first + u0 .., each of queries (below `each`) or keys
    const unsigned int row_bytes = (unsigned int)D * 2u;
    const int col = lane & 15, g = lane >> 4, r8 = lane >> 3;
    // piece p of row r of eight lands in slot p ^ (r >> 1), with 4 on top in every other group of eight rows: 16 rows read at one
    // piece touch 16 different 16-byte bank groups
    const int piece[2] = {((lane & 7) ^ (r8 >> 1)) * 16, ((lane & 7) ^ (4 + (r8 >> 1))) * 16};
    char *const ring = lds + w * kAdWaveBytes;
    unsigned int aoff[U], xoff[XT];
    bool key[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int u = first + min(u0 + i, total - 1);    // (units past the end repeat the last one, unused)
        key[i] = u >= each;
        aoff[i] = (unsigned int)((u - (key[i] ? each : 0)) * 8 + r8) * row_bytes + piece[i & 1];
    }
#pragma unroll
    for (int i = 0; i < XT; ++i) xoff[i] = (unsigned int)min(c0 + 8 * i + r8, Tn - 1) * row_bytes + piece[i & 1];
    const int n_mine = (D / 64 - w + WAVES - 1) / WAVES;                 // blocks of this wave: w, w + WAVES, ..
#if defined(__HIP_DEVICE_COMPILE__)
    auto base = [&](const char *from, size_t at) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from + at), 0, -1, 0x00020000); };
    const auto x_rs = base(x, (size_t)b * Tn * row_bytes);
    const auto q_rs = base(a_q != nullptr ? a_q : a_k, (size_t)a * R * row_bytes);
    const auto k_rs = base(a_k != nullptr ? a_k : a_q, (size_t)a * R * row_bytes);
#endif
    auto fetch = [&](int s, int at) {
#if defined(__HIP_DEVICE_COMPILE__)
        const unsigned int off = (unsigned int)(w + s * WAVES) * 128u;
        auto load = [&](__amdgpu_buffer_rsrc_t rs, unsigned int from, int i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(ring + at * kBytes + i * 1024), 16, (int)from, 0, 0, 0);
        };
#pragma unroll
        for (int i = 0; i < U; ++i) load(key[i] ? k_rs : q_rs, aoff[i] + off, i);
#pragma unroll
        for (int i = 0; i < XT; ++i) load(x_rs, xoff[i] + off, U + i);
#endif
    };
    // all requests but those of the `younger` last blocks have landed
    auto landed = [&](int younger) {
#if defined(__HIP_DEVICE_COMPILE__)
        if (younger >= N - 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((N - 1) * kLoads) : "memory");
        else
            unroll<N - 1>([&](auto m) {
                if (younger == m.value) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(m.value * kLoads) : "memory");
            });
#endif
    };
    f32x4 acc[NB][TT];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < N - 1; ++s)
        if (s < n_mine) fetch(s, s);
    int at = 0;
    for (int s = 0; s < n_mine; ++s) {
        if (s + N - 1 < n_mine) fetch(s + N - 1, at == 0 ? N - 1 : at - 1);
        landed(n_mine - 1 - s);
        const char *from = ring + at * kBytes;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            // (rows past an odd number of units are of no rank or token; of one unit the row itself is read again)
            const int slot = ((4 * i + g) ^ ((col >> 1) & 7)) << 4, slot8 = ((4 * i + g) ^ ((col & 7) >> 1)) << 4;
            Frag fa[NB], fx[TT];
#pragma unroll
            for (int j = 0; j < NB; ++j) fa[j].raw = *reinterpret_cast<const u32x4 *>(from + (j * 16 + (U == 1 ? col & 7 : col)) * 128 + (U == 1 ? slot8 : slot));
#pragma unroll
            for (int j = 0; j < TT; ++j) fx[j].raw = *reinterpret_cast<const u32x4 *>(from + (U * 8 + j * 16 + (XT == 1 ? col & 7 : col)) * 128 + (XT == 1 ? slot8 : slot));
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < TT; ++e) acc[j][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[j].bf, fx[e].bf, acc[j][e], 0, 0, 0);
        }
        at = at == N - 1 ? 0 : at + 1;
    }
    __syncthreads();
    f32x4 *const red = reinterpret_cast<f32x4 *>(lds);   // [wave][NB][TT][lane]
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) red[((w * NB + i) * TT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // lane l holds ranks 16 i + 4*(l/16) .. +3 of the group, of token l%16
    const float scale = scales != nullptr ? scales[a] : 1.f;
    for (int out = w; out < NB * TT; out += WAVES) {
        const int i = out / TT, j = out % TT, tok = c0 + j * 16 + col, u = u0 + 2 * i + (g >> 1);
        if (tok >= Tn || tok >= c0 + 8 * XT || 2 * i + (g >> 1) >= U || u >= total) continue;
        f32x4 sum = red[(i * TT + j) * 64 + lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += red[((v * NB + i) * TT + j) * 64 + lane];
        const int part = first + u >= each ? 1 : 0, rank = (first + u - part * each) * 8 + (g & 1) * 4;
        bf16x4 hi, mid, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Parts y = parts_of(scale * sum[e]);
            hi[e] = (__bf16)y.hi;
            mid[e] = (__bf16)y.mid;
            lo[e] = (__bf16)y.lo;
        }
        char *to = t + (((size_t)b * Tn + tok) * 2 + part) * (size_t)((R + 15) / 16 * kAdapterChunkBytes) + rank / 16 * kAdapterChunkBytes + rank % 16 * 2;
        *reinterpret_cast<bf16x4 *>(to) = hi;
        *reinterpret_cast<bf16x4 *>(to + 32) = mid;
        *reinterpret_cast<bf16x4 *>(to + 64) = lo;
    }
}

size_t adapter_row_bytes(int Tn, int R) { return (size_t)Tn * 2 * ((R + 15) / 16) * kAdapterChunkBytes; }

template <int U, int XT, int WAVES>
int launch_down(const char *x, const int32_t *ids, const char *a_q, const char *a_k, const float *scales, int n, int R, int B, int Tn, int D,
                char *t, hipStream_t stream)
{
    const int total = R / 8 * ((a_q ? 1 : 0) + (a_k ? 1 : 0)), groups = (total + U - 1) / U, tiles = (Tn + 8 * XT - 1) / (8 * XT);
    static DeviceFlags lds_allowed;
    const size_t lds = (size_t)WAVES * wave_bytes(WAVES);
    const auto kernel = adapter_down_kernel<U, XT, WAVES>;
    const hipError_t attr = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), lds, lds_allowed);
    if (attr != hipSuccess) return (int)attr;
    // A launch has less than 2^32 threads.  (A row has less than 2^32 bytes of at least 128 a token: less than 2^25 tokens, which fit.)
    const int most = (int)(0xffffffffll / (WAVES * 64) / groups / 8 * 8 / tiles);
    for (long long b = 0; b < B; b += most) {
        const long long n_tiles = (B - b < most ? B - b : most) * tiles, items = n_tiles * groups, grid = (n_tiles + 7) / 8 * 8 * groups;
        const int e = (int)launch_kernel(kernel, dim3((unsigned int)grid), dim3(WAVES * 64), lds, stream, KernelEvents{}, x + (size_t)b * Tn * D * 2,
                                         ids + b, a_q, a_k, scales, n, R, Tn, D, tiles, groups, (unsigned int)items,
                                         t + (size_t)b * adapter_row_bytes(Tn, R));
        if (e != (int)hipSuccess) return e;
    }
    return (int)hipSuccess;
}

}  // namespace

size_t adapter_workspace_bytes(int B, int Tn, int R) { return (B * adapter_row_bytes(Tn, R) + 255) / 256 * 256; }

int launch_adapter_down(const void *x_, const int32_t *ids, const void *a_q_, const void *a_k_, const float *scales, int n, int R, int B, int Tn,
                        int D, void *t_, hipStream_t stream)
{
    const char *x = static_cast<const char *>(x_), *a_q = static_cast<const char *>(a_q_), *a_k = static_cast<const char *>(a_k_);
    char *t = static_cast<char *>(t_);
    // Few tokens of a row: as many workgroups as there are eights of ranks and tokens, of sixteen waves, while that is a round of the chip
    // (8 rows x 37 tokens, width 9216, rank 8 of queries alone, with the projections 84.7 us; eight waves of 16 ranks x 16 tokens 87.4),
    // else two or four eights of ranks each, or sixteen tokens where a row has more (4 x 50 tokens, rank 64, 27.4 us instead of 31.4; 31 rows x 1
    // token, rank 128, 36.1 instead of 42.2).  Sixteen tokens and one eight of ranks are the faster while they are a round of the chip, width 4096,
    // rank 128: 4 x 32 tokens 5.0 us, 32 tokens and four eights 6.6; beyond one they are not: 8 x 64 17 and 8, 16 x 64 30 and 9, 64 x 64 115 and 25.
    const long long eights = (long long)B * ((Tn + 7) / 8) * (R / 8) * ((a_q ? 1 : 0) + (a_k ? 1 : 0));
    auto go = [&](auto u, auto xt, auto waves) {
        return launch_down<decltype(u)::value, decltype(xt)::value, decltype(waves)::value>(x, ids, a_q, a_k, scales, n, R, B, Tn, D, t, stream);
    };
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 2> two{};
    constexpr std::integral_constant<int, 4> four{};
    constexpr std::integral_constant<int, 16> sixteen{};
    if (Tn <= 8) return eights <= 256 ? go(one, one, sixteen) : eights <= 512 ? go(two, one, sixteen) : go(four, one, sixteen);
    if (Tn <= 64) return eights <= 256 ? go(one, one, sixteen) : go(one, two, sixteen);
    return go(four, four, four);
}

}  // namespace chai
