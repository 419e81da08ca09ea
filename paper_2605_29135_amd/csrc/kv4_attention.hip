// kv4_attention.hip -- attention over the 4-bit cache (layout in kv4.h), one or many tokens per sequence.
//
// With K = s_g u + m_g per group g of 64 dims, q . K_p = sum_g s_gp (q_g . u_gp) + m_gp (sum of q_g), and the value
// side is sum_p (P_p s_gp) (u_p - 8) + P_p (m_gp + 8 s_gp).  Four bits at the bottom of an fp16 are the subnormal
// u 2^-24 (at bits 4-7: 16 u 2^-24, the 16 taken out of the other operand), so one bit operation makes two operands
// of a matrix product, and where they have to be normal or centred one packed fma does it; every product is exact.
// Scores are formed transposed (positions x rows), so that a lane holds one row's probabilities of the positions that
// are its operand of the value product (they stay in registers), and the outputs as dims x rows, so that a row's
// running maximum and sum belong to its lane.
//
// fp16 reaches far enough because both other operands are scaled by powers of two: a row's query so that its
// largest element is in [2^14, 2^15), the values' scales so that the largest the wave has met is at most 2^15
// (the outputs so far are scaled along when that grows).  Queries: bf16 ones are exact, fp32 ones are two terms
// (2^-22 of the row's largest).  P s: rounded to fp16 (2^-11, bf16 tensors) or two terms (2^-22).  What multiplies
// the bases is fp32.
//
// A row is a (token, query head of the group) pair; a wave takes NT tiles of 16 rows over every fourth block
// of 32 positions, and the block's waves join their (max, sum, output) through LDS.  With few rows the
// positions are split over more blocks (grid), whose partial results a second launch joins.
//
// Bound: with few rows the cache's bytes, 1.125 d per position and key/value head.  Measured (kernel, then join; inputs
// that change from pass to pass, more than the last-level cache holds): one token of 64 heads over 131071 positions of 8
// heads of 128, bf16, 32.6 + 4.9 us (151 MB, 4.6 TB/s of the 7.2 that a large read reaches); 16 sequences of up to 16384,
// 40.8 + 4.8 us (188 MB, 4.6 TB/s); one token of 32 heads over 4096 positions of 4 heads, fp32, 7.2 + 3.9 us, which is
// latency (each wave has one block of positions, loaded for both of the places that the code has).  One block of
// positions in flight per wave instead of two: 37.8 us for the 37.1 of the first, 47.2 for the 45.8 of the second.  Rows
// that fill only half of a tile (up to 8) share the lanes between a block's two tiles of positions, which halves the lane
// arithmetic: 46.0 us for the 16 sequences, 48.3 without.
#include "device_common.h"
#include "internal.h"
#include "kv4.h"

#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

using namespace kv4;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kAttWaves = 4, kAttBlock = 64 * kAttWaves;
// Blocks that fill the device, where rows and heads alone give fewer: one token of 64 heads over 131071 positions of
// 8 heads takes 37.1 us (with the join) with 512, 39.9 with 256, 41.0 with 768 and 42.2 with 1024.
constexpr int kTarget = 512;

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma(f16x8 a, f16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// The eight codes of a word as fp16: u 2^-24 (elements 0, 1, 4, 5) and 16 u 2^-24 (elements 2, 3, 6, 7).
__device__ __forceinline__ f16x8 raw_codes(uint32_t w) {
    constexpr uint32_t L = 0x000F000Fu, H = 0x00F000F0u;
    const uint32_t v = w >> 8;
    return __builtin_bit_cast(f16x8, make_uint4(w & L, w & H, v & L, v & H));
}
constexpr bool high_code(int i) { return i & 2; }
// Keys.  A subnormal operand's products are aligned as if it were 2^-14: sums lose up to 10 of their bits, which the
// scores of bf16 queries can spare (about 1e-5); fp32 queries meet u 2^-9 and 16 u 2^-9.
template <bool F32> constexpr int kKeyExp = F32 ? -9 : -24;
template <bool F32>
__device__ __forceinline__ f16x8 key_codes(uint32_t w) {
    const f16x8 u = raw_codes(w);
    return F32 ? u * _Float16(0x1p15f) : u;
}
// Values: (u - 8) 2^-9.  Sums of P s u over a long cache would only grow, while what is left
// of them after P m is the mean of values of either sign (of 131071 positions: hundreds of times less).
constexpr int kValueExp = -9;
__device__ __forceinline__ f16x8 value_codes(uint32_t w) {
    constexpr _Float16 m = 0x1p15f, n = 0x1p11f, a = -0x1p-6f;
    return raw_codes(w) * f16x8{m, m, n, n, m, m, n, n} + f16x8{a, a, a, a, a, a, a, a};
}

__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // round to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {__bf16(lo), __bf16(hi)};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ f16x2 pack_f16(float lo, float hi) {
    const f16x2 v = {_Float16(lo), _Float16(hi)};
    return v;
}
__device__ __forceinline__ f16x8 join8(f16x2 a, f16x2 b, f16x2 c, f16x2 d) {
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// a b, rounded: what is subtracted from it later meets the same number (contracted into an fma it would be another).
__device__ __forceinline__ float product(float a, float b) {
#pragma clang fp contract(off)
    float v = a * b;
    asm("" : "+v"(v));
    return v;
}
// Eight values as TERMS fp16 operands, the second rounding what the first leaves.
template <int TERMS>
__device__ __forceinline__ void split(const float (&x)[8], f16x8 (&t)[TERMS]) {
    f16x2 h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = pack_f16(x[2 * e], x[2 * e + 1]);
    t[0] = join8(h[0], h[1], h[2], h[3]);
    if constexpr (TERMS == 2) {
        f16x2 l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) l[e] = pack_f16(x[2 * e] - float(h[e][0]), x[2 * e + 1] - float(h[e][1]));
        t[1] = join8(l[0], l[1], l[2], l[3]);
    }
}

// From a row's scores as formed to log2 units: 2^e2 scales its query, `exp` is in its operands.  Held finite, so that a
// difference of scores times it is right at any size (0 stays 0, and what is far from 0 stays far).
__device__ __forceinline__ float row_unit(float scale, int exp) {
    return fminf(fmaxf(ldexpf(fabsf(scale), exp), 0x1p-126f), 0x1p126f);
}
// Scores from here on (log2 units) are far: a product of a score and the row's unit, rounded, is then off by so much
// (2^-4 at 2^20) that exponentials relative to it leave fp16's range, and is itself infinite further on.  A row that
// meets one takes its exponentials of differences of scores instead, one operation more for each.
constexpr float kFar = 0x1p20f;
__device__ __forceinline__ bool is_far(float off) { return !(fabsf(off) < kFar); }

// What f makes of v over the four lanes (n, 0..3).
template <typename F>
__device__ __forceinline__ float over_c(float v, F f) {
    auto pair = [](auto r) { return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1])); };
    float2 u = pair(__builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    v = f(u.x, u.y);
    u = pair(__builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return f(u.x, u.y);
}
__device__ __forceinline__ float max_over_c(float v) {
    return over_c(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_over_c(float v) {
    return over_c(v, [](float a, float b) { return a + b; });
}
// The value of lane n ^ 8.
template <typename T>
__device__ __forceinline__ T other_half(T v) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xF, 0xF, false));
}
// Sums over the lanes up to this one.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
#define SCAN(CTRL, ROWS) v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, ROWS, 0xF, true))
    SCAN(0x111, 0xF);  // row_shr:1
    SCAN(0x112, 0xF);
    SCAN(0x114, 0xF);
    SCAN(0x118, 0xF);
    SCAN(0x142, 0xA);  // row_bcast:15 into rows 1 and 3
    SCAN(0x143, 0xC);  // row_bcast:31 into rows 2 and 3
#undef SCAN
    return v;
}

struct AttendArgs {
    const void *q;
    void *out;
    const uint8_t *cache;
    float *part;  // [unit][head][tile][16 NT rows][d + 4]: unnormalised output, maximum, sum, the row's unit (row_unit)
    long long q_stride, out_stride;
    int n_heads, n_kv, group, window;
    int target;  // splits of a whole batch (0: every sequence in one piece)
    int least;   // blocks of positions that a piece has at least; the rest come in multiples of `unit`
    int unit;
    int tiles;   // row tiles of the largest sequence
    float scale;  // times log2(e)
    Batch batch;
    int *err;
};

// The first position that some token of the sequence sees.
__device__ __forceinline__ int first_seen(const Seq &s, int window) {
    return window ? max(0, s.len - s.n - window + 1) : 0;
}
// Blocks of positions that a sequence's tokens see.
__device__ __forceinline__ int seen_blocks(const Seq &s, int window) {
    if (s.n == 0 || s.len == 0) return 0;
    return (s.len - 1) / kPos + 1 - first_seen(s, window) / kPos;
}

// The split of a batch: sequences are cut into pieces of `chunk` blocks of positions, at least `least`, so
// that there are about `target` of them in all; a sequence has at least one piece.  Every wave works it out for
// itself.  by_unit: which piece is number `want`; otherwise, the pieces of sequence `want`.
struct Piece {
    Seq s;
    int seq, split, chunk;
    int first, count;  // of the sequence's pieces (count 0: there is no such piece)
};
__device__ __forceinline__ Piece find_piece(const AttendArgs &a, int want, bool by_unit, int *err) {
    const Batch &b = a.batch;
    const int window = a.window, target = a.target;
    const int lane = threadIdx.x & 63;
    uint32_t total = 0;  // (a batch that is split has fewer than kTarget sequences of at most 2^21 blocks)
    Seq s{0, 0, 0, false};
    int nb = 0;
    auto look = [&](int base) {
        s = Seq{0, 0, 0, false};
        if (base + lane < b.n_seq) s = sequence(b, base + lane);
        nb = seen_blocks(s, window);
    };
#pragma unroll 1
    for (int base = 0; base < b.n_seq; base += 64) {
        look(base);
        if (err && s.bad) atomicOr(err, kErrRange);
        total += uint32_t(__builtin_amdgcn_readlane(int(wave_scan(uint32_t(nb))), 63));
    }
    Piece p{};
    p.chunk = max(int((total + uint32_t(target) - 1) / uint32_t(target)), a.least);
    p.chunk = (p.chunk + a.unit - 1) & -a.unit;
    // (pieces rounded up may be more than run together, and the last few would take as long again: somewhat larger ones
    // that do are better.  16 sequences of 4822 to 16384 positions: 54.0 us without, 45.8 with.  More sequences than lanes
    // would have to be read again for every size tried.)
    if (b.n_seq > 1 && b.n_seq <= 64) {
        int chunk = p.chunk;
#pragma unroll 1
        for (int k = 1; k <= 8; ++k) {
            const int count = s.n ? max(1, (nb + chunk - 1) / chunk) : 0;
            if (__builtin_amdgcn_readlane(int(wave_scan(uint32_t(count))), 63) <= target) {
                p.chunk = chunk;
                break;
            }
            chunk = (p.chunk + p.chunk * k / 8 + a.unit - 1) & -a.unit;
        }
    }
    int before = 0;
#pragma unroll 1
    for (int base = 0; base < b.n_seq; base += 64) {
        if (b.n_seq > 64) look(base);
        const int count = s.n ? max(1, (nb + p.chunk - 1) / p.chunk) : 0;
        const int upto = int(wave_scan(uint32_t(count))), first = before + upto - count;
        const bool mine = by_unit ? want >= first && want < first + count : base + lane == want;
        const unsigned long long hit = __ballot(mine);
        if (hit) {
            const int l = __builtin_amdgcn_readfirstlane(__ffsll(hit) - 1);
            p.seq = base + l;
            p.first = __builtin_amdgcn_readlane(first, l);
            p.count = __builtin_amdgcn_readlane(count, l);
            p.s.t0 = __builtin_amdgcn_readlane(s.t0, l);
            p.s.n = __builtin_amdgcn_readlane(s.n, l);
            p.s.len = __builtin_amdgcn_readlane(s.len, l);
            p.split = by_unit ? want - p.first : 0;
            return p;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return p;
}

// This block's piece: grid (row tiles, key/value head, sequence), or (key/value head, row tiles, pieces), where the pieces
// that there are not come last (among the others they would leave some of the eight dies with more blocks than run
// together).
__device__ __forceinline__ Piece this_piece(const AttendArgs &a, int tile, int *err) {
    if (a.target) return find_piece(a, blockIdx.z, true, blockIdx.z == 0 ? err : nullptr);
    Piece p{};
    p.seq = blockIdx.z;
    p.count = 1;
    p.s = sequence(a.batch, p.seq);
    if (p.s.bad && err && (threadIdx.x & 63) == 0) atomicOr(err, kErrRange);
    return p;
}
// Blocks of positions (first, end): those that some of the rows sees, the piece's share of them.
__device__ __forceinline__ int2 tile_blocks(const AttendArgs &a, const Piece &piece, int row, int row_end) {
    const Seq &s = piece.s;
    const int p_first = s.len - s.n + row / a.group, p_last = s.len - s.n + (row_end - 1) / a.group;
    const int b_first = first_seen(s, a.window) / kPos;
    const int t_first = a.window ? max(0, p_first - a.window + 1) / kPos : 0, t_end = p_last < 0 ? 0 : p_last / kPos + 1;
    return make_int2(max(t_first, b_first + piece.split * piece.chunk),
                     piece.split == piece.count - 1 ? t_end : min(t_end, b_first + (piece.split + 1) * piece.chunk));
}

template <bool F32>
__device__ __forceinline__ void store4(void *out, size_t at, float4 v) {
    if constexpr (F32) *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = v;
    else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// grid: (row tiles, key/value head, sequence), or with a target (key/value head, row tiles, pieces).
// HALF: at most 8 rows.  They fill columns 0-7 and again 8-15, and lane (n, c) takes row n % 8's scores of the
// positions of tile n / 8 alone: half the arithmetic per lane; the probabilities of tile 1 are handed to the lanes
// of column n - 8 as operands.
template <int NG, int NT, bool F32, bool HALF>
__global__ __launch_bounds__(kAttBlock, NG * NT <= 2 ? 2 : 1) void kv4_attend_kernel(AttendArgs a) {
    constexpr int d = NG * kGroup, TERMS = F32 ? 2 : 1, ROWS = HALF ? 8 : 16, PP = HALF ? 4 : 8;
    constexpr int UB = NG <= 2 && NT == 1 && (HALF || !F32 || NG == 1) ? 2 : 1;  // blocks of positions at a time
    static_assert(!HALF || NT == 1);
    __shared__ float4 out_sh[kAttWaves][ROWS][d / 4 + 1];
    __shared__ float max_sh[kAttWaves][ROWS], sum_sh[kAttWaves][ROWS], unit_sh[ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4;
    const int half = HALF ? n >> 3 : 0, n_row = HALF ? n & 7 : n;
    const int tile = a.target ? blockIdx.y : blockIdx.x, h = a.target ? blockIdx.x : blockIdx.y;
    const Piece piece = this_piece(a, tile, tile == 0 && h == 0 && threadIdx.x < 64 ? a.err : nullptr);
    if (piece.count == 0) return;
    const Seq &s = piece.s;
    const int G = a.group, rows = s.n * G, row0 = tile * ROWS * NT;
    if (row0 >= rows) return;
    const int p_first = s.len - s.n + row0 / G;                               // position of the tile's first row
    const int p_last = s.len - s.n + min(s.n - 1, (row0 + ROWS * NT - 1) / G);  // of its last row
    const int2 range = tile_blocks(a, piece, row0, min(row0 + ROWS * NT, rows));
    const int b0 = range.x, b1 = range.y, p_seen = first_seen(s, a.window);
    const uint8_t *seq = a.cache + (size_t(piece.seq) * a.n_kv + h) * (a.batch.max_pos / kPos) * block_bytes(d);

    // A block's operands as they lie in the cache.  Keys and values are loaded one block ahead, each as soon as
    // the present block's have been used; past the wave's last block the last one is loaded again.
    uint4 kc[UB][NG], vc[UB][NG];
    uint32_t ks[UB][NG][PP / 2], vs[UB][NG][PP / 2], vm[UB][NG][PP / 2], km[UB];
    auto load_pairs = [&](const uint8_t *p, uint32_t (&v)[PP / 2]) __attribute__((always_inline)) {
        if constexpr (HALF) {
            const uint2 u = *reinterpret_cast<const uint2 *>(p + c * 16 + half * 8);
            v[0] = u.x, v[1] = u.y;
        } else {
            const uint4 u = dev::load16(p + c * 16);
            v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
        }
    };
    // (the u-th of the wave's next blocks, the first again where there is none)
    auto block_at = [&](int b, int u) { return seq + size_t(b + u * kAttWaves < b1 ? b + u * kAttWaves : b) * block_bytes(d); };
    auto load_k = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UB; ++u) {
            const uint8_t *block = block_at(b, u);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                kc[u][g] = dev::load16(block + k_codes(d) + g * 1024 + lane * 16);
                load_pairs(block + k_scales(d) + g * 64, ks[u][g]);
            }
            km[u] = *reinterpret_cast<const uint32_t *>(block + k_bases(d) + min(c, NG - 1) * 64 + n * 4);
        }
    };
    auto load_v = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UB; ++u) {
            const uint8_t *block = block_at(b, u);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                vc[u][g] = dev::load16(block + v_codes(d) + g * 1024 + lane * 16);
                load_pairs(block + v_scales(d) + g * 64, vs[u][g]);
                load_pairs(block + v_bases(d) + g * 64, vm[u][g]);
            }
        }
    };
    // (a row past the last repeats it and is not stored)
    constexpr int QV = F32 ? 2 : 1;  // 16-byte loads per 8 elements of q
    uint4 qraw[NT][2 * NG][QV];
    auto row_of = [&](int t) { return min(row0 + 16 * t + n_row, rows - 1); };
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = row_of(t), i = row / G;
        const size_t at = size_t(s.t0 + i) * a.q_stride + size_t(h * G + row - i * G) * d + 8 * c;
#pragma unroll
        for (int j = 0; j < 2 * NG; ++j)
#pragma unroll
            for (int e = 0; e < QV; ++e)
                qraw[t][j][e] = dev::load16(static_cast<const uint8_t *>(a.q) + (at + 32 * j) * (F32 ? 4 : 2) + 16 * e);
    }
    // (no branch: a wave without a block reads the cache's first, and uses none of it)
    {
        const int b = b0 + wave < b1 ? b0 + wave : 0;
        load_k(b);
        load_v(b);
    }
    __builtin_amdgcn_sched_barrier(0);

    // The tile's rows: their queries as operands (k = dims), their last visible position.
    int last[NT];
    float zs[NT];  // from a score as formed to log2 units
    f16x8 bq[NT][2 * NG][TERMS];
    bf16x8 bm[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        last[t] = s.len - s.n + row_of(t) / G;
        float x[2 * NG][8], top = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * NG; ++j) {
            const uint4 u = qraw[t][j][0], v = qraw[t][j][QV - 1];
            if constexpr (F32) {
                const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = __uint_as_float(w[e]);
            } else {
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[j][2 * e] = low_half(w[e]);
                    x[j][2 * e + 1] = high_half(w[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[j][e]));
        }
        top = max_over_c(top);
        // 2^e takes the row's largest element to [2^14, 2^15).  (From 2^103 on, which the limits of a call leave
        // out, it would not fit fp16; an infinity or NaN stays one.)
        int e2 = 0;
        if (top > 0.f && top < INFINITY) e2 = min(max(14 - ilogbf(top), -88), 148);
        zs[t] = row_unit(a.scale, -kKeyExp<F32> - e2);
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float sg = 0.f;
#pragma unroll
            for (int j = 2 * g; j < 2 * g + 2; ++j) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = ldexpf(a.scale < 0.f ? -x[j][e] : x[j][e], e2);
                    sg += y;
                    x[j][e] = high_code(e) ? y * 0.0625f : y;
                }
                split<TERMS>(x[j], bq[t][j]);
            }
            sg = sum_over_c(sg);
            sum = c == g ? sg : sum;
        }
        // The bases' product: elements (c, 0..2) are the sum of q over group c as three bf16 terms.
        sum = ldexpf(sum, kKeyExp<F32>);
        const uint32_t w1 = bf16_rne(sum);
        const float r1 = sum - bf16_float(w1);
        const uint32_t w2 = bf16_rne(r1);
        const uint32_t w3 = bf16_rne(r1 - bf16_float(w2));
        bm[t] = __builtin_bit_cast(bf16x8, make_uint4(w1 | (w2 << 16), w3, 0, 0));
    }

    // A row's sums hold 2^boost P with P = exp2(score - off), off the largest score so far, in log2 units; 2^boost
    // takes the largest value scale so far to about 2^15.  When either changes, the sums so far are scaled along.
    // (An off with the boost in it would cost P 4 bits: the exponent is rounded at its own size.)
    floatx4 acc[NT][4 * NG];  // sum of P s (u - 8) (dims x rows), times 2^(boost + kValueExp)
    float add[NT][NG];        // sum of P (m + 8 s), this lane's positions
    float mx[NT], off[NT], sum[NT];
    bool far[NT], any_far = false;  // (of the row; of any: P and the sums are relative to mx itself, off is 0)
    uint32_t top_s = 0;  // largest bf16 of the exponent of the largest value scale so far
    int boost = 0;
    float boost_f = 1.f;  // 2^boost
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        mx[t] = -INFINITY;
        off[t] = sum[t] = 0.f;
        far[t] = false;
#pragma unroll
        for (int i = 0; i < 4 * NG; ++i) acc[t][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < NG; ++g) add[t][g] = 0.f;
    }
    // The wave's blocks b, b + kAttWaves, ... (U of them), whose operands are loaded; `next`: what to load meanwhile.
    auto step = [&](auto blocks, int b, int next) __attribute__((always_inline)) {
        constexpr int U = decltype(blocks)::value;
        // ---- scores
        float p[NT][U][PP];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            floatx4 z0[NT], y0[NT][NG];
#pragma unroll
            for (int tau = 0; tau < 2; ++tau) {
                const uint32_t m2 = tau ? (km[u] & 0xffff0000u) | (km[u] >> 16) : (km[u] << 16) | (km[u] & 0xffffu);
                const bf16x8 ma = __builtin_bit_cast(bf16x8, make_uint4(m2, m2, m2, m2));
                f16x8 kf[2 * NG];
#pragma unroll
                for (int j = 0; j < 2 * NG; ++j) {
                    const int w = tau * 2 * NG + j;
                    kf[j] = key_codes<F32>(reinterpret_cast<const uint32_t *>(&kc[u][w / 4])[w % 4]);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    floatx4 z = mfma(ma, bm[t], floatx4{0.f, 0.f, 0.f, 0.f}), y[NG];
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        y[g] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                            for (int j = 2 * g; j < 2 * g + 2; ++j) y[g] = mfma(kf[j], bq[t][j][k], y[g]);
                    }
                    if constexpr (HALF) {
                        if (tau == 0) {
                            z0[t] = z;
#pragma unroll
                            for (int g = 0; g < NG; ++g) y0[t][g] = y[g];
                            continue;
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            z[r] = half ? z[r] : z0[t][r];
#pragma unroll
                            for (int g = 0; g < NG; ++g) y[g][r] = half ? y[g][r] : y0[t][g][r];
                        }
                    }
                    constexpr int stride = HALF ? 0 : 4;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            const uint32_t w = ks[u][g][(stride * tau + r) / 2];
                            z[r] = fmaf(r & 1 ? high_half(w) : low_half(w), y[g][r], z[r]);
                        }
                        p[t][u][stride * tau + r] = z[r];
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (what is next waits for the values: it stays behind the keys' loads)
        load_k(next);
        __builtin_amdgcn_sched_barrier(0);
        // ---- softmax
        const int past = b + (U - 1) * kAttWaves;  // the last of the blocks
        if (past * kPos + kPos > s.len || b * kPos < p_seen) {
            // Positions past the last, and those in front of the first that some token sees, may never have been
            // written and hold anything: their probabilities are 0, and 0 times what lies there has to be 0.
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < PP / 2; ++i) {
                    uint32_t keep = 0;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int k = 2 * i + e, at = (b + u * kAttWaves) * kPos + 16 * (half + (k >> 2)) + 4 * c + (k & 3);
                        keep |= at < s.len && at >= p_seen ? 0xffffu << (16 * e) : 0u;
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        vs[u][g][i] &= keep;
                        vm[u][g][i] &= keep;
                    }
                }
        }
        u16x2 most = {0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int i = 0; i < PP / 2; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, vs[u][g][i]));
        const uint32_t most_s = max(most[0], most[1]);
        const bool scales_rose = __any(most_s > top_s);
        float rise = 1.f;
        if (scales_rose) {
            const int e = int(dev::wave_reduce_u32<true>(most_s) >> 7), was = boost;
            top_s = (uint32_t(e) << 7) | 0x7fu;
            boost = min(141 - e, 60);  // (sums of bases up to 2^40 over up to 2^26 positions stay finite)
            boost_f = ldexpf(1.f, boost);
            rise = ldexpf(1.f, min(boost - was, 126));  // (it rises from its start only: the sums are still zeros)
        }
        const bool full = past * kPos + kPos - 1 <= p_first && (!a.window || b * kPos > p_last - a.window);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (!full) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < PP; ++k) {
                        const int at = (b + u * kAttWaves) * kPos + 16 * (half + (k >> 2)) + 4 * c + (k & 3);
                        if (at > last[t] || (a.window && at <= last[t] - a.window)) p[t][u][k] = -INFINITY;
                    }
            }
            float top = p[t][0][0];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < PP; ++k) top = fmaxf(top, p[t][u][k]);
            if constexpr (HALF) top = fmaxf(top, other_half(top));
            top = max_over_c(top);
            const float was = mx[t], now = fmaxf(was, top);
            if (scales_rose || any_far || __any(now > was)) {
                float to = now == -INFINITY ? 0.f : product(now, zs[t]), fall = off[t] - to;
                any_far |= __any(is_far(to));
                if (__builtin_expect(any_far, 0)) {
                    if (is_far(to) || far[t]) {
                        fall = fmaf(was - now, zs[t], far[t] ? 0.f : fmaf(-was, zs[t], off[t]));
                        far[t] = true;
                        to = 0.f;
                    }
                    const float from = far[t] ? now : 0.f;
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int k = 0; k < PP; ++k) p[t][u][k] -= from;
                }
                const float f = was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fall) * rise;
                mx[t] = now;
                off[t] = to;
                sum[t] *= f;
#pragma unroll
                for (int i = 0; i < 4 * NG; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][i][r] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g) add[t][g] *= f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < PP; ++k) {
                    p[t][u][k] = __builtin_amdgcn_exp2f(fmaf(p[t][u][k], zs[t], -off[t])) * boost_f;
                    sum[t] += p[t][u][k];
                }
        }
        // ---- values
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                f16x8 vf[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) vf[i] = value_codes(reinterpret_cast<const uint32_t *>(&vc[u][g])[i]);
                float sf[PP], mf[PP];
#pragma unroll
                for (int k = 0; k < PP; ++k) {
                    const uint32_t sw = vs[u][g][k / 2], mw = vm[u][g][k / 2];
                    sf[k] = k & 1 ? high_half(sw) : low_half(sw);
                    mf[k] = fmaf(8.f, sf[k], k & 1 ? high_half(mw) : low_half(mw));
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float y[8];
                    f16x8 bs[TERMS];
#pragma unroll
                    for (int k = 0; k < PP; ++k) {
                        // (two terms: both have to see one rounded product, not one of them a fused conversion)
                        y[k] = F32 ? product(p[t][u][k], sf[k]) : p[t][u][k] * sf[k];
                        add[t][g] = fmaf(p[t][u][k], mf[k], add[t][g]);
                    }
                    if constexpr (HALF) {
                        f16x2 lo[2][TERMS];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            lo[e][0] = pack_f16(y[2 * e], y[2 * e + 1]);
                            if constexpr (TERMS == 2)
                                lo[e][1] = pack_f16(y[2 * e] - float(lo[e][0][0]), y[2 * e + 1] - float(lo[e][0][1]));
                        }
#pragma unroll
                        for (int k = 0; k < TERMS; ++k)
                            bs[k] = join8(lo[0][k], lo[1][k], other_half(lo[0][k]), other_half(lo[1][k]));
                    } else {
                        split<TERMS>(y, bs);
                    }
#pragma unroll
                    for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[t][4 * g + i] = mfma(vf[i], bs[k], acc[t][4 * g + i]);
                }
            }
        __builtin_amdgcn_sched_barrier(0);
        load_v(next);
    };
    int b = b0 + wave;
#pragma unroll 1
    for (; b + (UB - 1) * kAttWaves < b1; b += UB * kAttWaves)
        step(std::integral_constant<int, UB>(), b, b + UB * kAttWaves < b1 ? b + UB * kAttWaves : b);
    if (UB == 2 && b < b1) step(std::integral_constant<int, 1>(), b, b);

    // Join the waves, one tile of rows at a time.
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // (relative to the largest score itself: its product with the unit, to which the sums are, is rounded)
        const float rel = far[t] || mx[t] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(fmaf(-mx[t], zs[t], off[t]));
        float l = sum_over_c(sum[t]);
        if constexpr (HALF) l += other_half(l);
        if (t) __syncthreads();
        if (c == 0 && !half) {
            max_sh[wave][n] = mx[t];
            sum_sh[wave][n] = ldexpf(l * rel, -boost);
            if (wave == 0) unit_sh[n] = zs[t];
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float m = sum_over_c(add[t][g]);
            if constexpr (HALF) m += other_half(m);
            m = ldexpf(m, -boost);
            const int e = -boost - kValueExp;
            if (!half)
#pragma unroll
                for (int i = 4 * g; i < 4 * g + 4; ++i)
                    out_sh[wave][n][4 * i + c] =
                        make_float4((ldexpf(acc[t][i][0], e) + m) * rel, (ldexpf(acc[t][i][1], e) + m) * rel,
                                    (ldexpf(acc[t][i][2], e) + m) * rel, (ldexpf(acc[t][i][3], e) + m) * rel);
        }
        __syncthreads();
#pragma unroll 1
        for (int idx = threadIdx.x; idx < ROWS * (d / 4); idx += kAttBlock) {
            const int r = idx / (d / 4), i4 = idx % (d / 4), row = row0 + 16 * t + r;
            if (row >= rows) continue;
            float M = max_sh[0][r];
#pragma unroll
            for (int w = 1; w < kAttWaves; ++w) M = fmaxf(M, max_sh[w][r]);
            float S = 0.f;
            const float unit = unit_sh[r];
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kAttWaves; ++w) {
                // (a wave that saw nothing of the row has the maximum -inf and the sum 0; one whose scores are
                // all NaN has the sum NaN, which stays)
                const float f = max_sh[w][r] == -INFINITY && sum_sh[w][r] == 0.f ? 0.f : __builtin_amdgcn_exp2f((max_sh[w][r] - M) * unit);
                const float4 u = out_sh[w][r][i4];
                S = fmaf(f, sum_sh[w][r], S);
                v.x = fmaf(f, u.x, v.x);
                v.y = fmaf(f, u.y, v.y);
                v.z = fmaf(f, u.z, v.z);
                v.w = fmaf(f, u.w, v.w);
            }
            if (piece.count > 1) {
                float *o = a.part + ((size_t(piece.first + piece.split) * a.n_kv + h) * a.tiles * (ROWS * NT) + row) * (d + 4);
                *reinterpret_cast<float4 *>(o + 4 * i4) = v;
                if (i4 == 0) *reinterpret_cast<float4 *>(o + d) = make_float4(M, S, unit, 0.f);
                continue;
            }
            const float inv = S == 0.f ? 0.f : 1.f / S;  // (a row that sees nothing: 0)
            v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
            store4<F32>(a.out, size_t(s.t0 + row / G) * a.out_stride + size_t(h * G + row % G) * d + 4 * i4, v);
        }
    }
}

// ---- many rows (prompts), bf16 tensors -------------------------------------------------------------------------
//
// Where a block of positions meets hundreds of rows the arithmetic per score counts, not the bytes: the waves of a
// block turn the codes of 64 positions into fp16 keys and values once (2^-11; scaled by powers of two, 2^6 the
// largest) and share them through LDS in the operands' order, and a score costs an fma, an exponential, a share
// of a maximum and of a conversion.  Two buffers: the next positions' codes are loaded before the present ones are
// used and turned after.  The sums of P come from the matrix cores too.
//
// Bound: the chain of a step (operands from LDS, scores, softmax, products, a barrier), about 2.5 us for 64 positions at
// either block size, and blocks of unequal length.  2048 tokens of 32 heads of 128 over 8192 positions: 329 us (after some
// 20 ms of work; 373 for the first launches of an idle device, whose clock still rises), 0.73 PFLOP/s (1.22 for a large
// bf16 product); the matrix cores are busy 30 % of the time and lanes issue 45 % of it (counters); its 256 blocks are one
// per unit and walk 97 to 128 steps, so 12 % is idle behind the shorter ones.  With heads of 256, 16 of them: 365 us,
// 0.66.  Two groups of waves a phase apart: 401 us for the 366 that the first form took.
constexpr int prompt_tiles(int d) { return d <= 128 ? 2 : 1; }  // row tiles of 16 per wave: what its registers hold

// A barrier for what the block's waves pass one another through LDS; loads in flight stay so.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// The power of two that takes values of at most |m| + 15 s below 2^6: m, s pairs of bf16, L per lane (s >= 0).
template <int L>
__device__ __forceinline__ int held_exponent(const uint32_t (&m)[L], const uint32_t (&s)[L]) {
    // 2 max(|m|, 16 s) is no less; bf16 bits compare as numbers, and four exponents more are times 16
    u16x2 v = {0, 0};
#pragma unroll
    for (int l = 0; l < L; ++l) {
        v = __builtin_elementwise_max(v, __builtin_bit_cast(u16x2, m[l] & 0x7fff7fffu));
        v = __builtin_elementwise_max(v, __builtin_bit_cast(u16x2, s[l] + 0x02000200u));
    }
    int top = max(int(v[0]), int(v[1]));
#define ROW_MAX(CTRL) top = max(top, __builtin_amdgcn_update_dpp(0, top, CTRL, 0xF, 0xF, true))
    ROW_MAX(0xB1);
    ROW_MAX(0x4E);
    ROW_MAX(0x141);
    ROW_MAX(0x140);
#undef ROW_MAX
    const int all = max(max(__builtin_amdgcn_readlane(top, 0), __builtin_amdgcn_readlane(top, 16)),
                        max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)));
    return min(131 - (all >> 7), 100);  // (below 2^(exponent - 127 + 2))
}

// grid: (row tiles, key/value head, sequence), or with a target (key/value head, row tiles, pieces); WAVES x 16 NT rows
// per block.
template <int NG, int WAVES>
__global__ __launch_bounds__(64 * WAVES, NG <= 2 ? 2 : WAVES / 4) void kv4_prompt_kernel(AttendArgs a) {
    constexpr int d = NG * kGroup, NT = prompt_tiles(d), ROWS = 16 * NT * WAVES;
    constexpr int FRAGS = 8 * NG;           // operands (1 KiB) of two blocks' keys, and of their values
    constexpr int WORDS = 16 * NG / WAVES;  // words of codes per lane that a wave turns
    constexpr int SPLIT = WAVES / 4;        // waves that share one block's keys or values
    constexpr int LIM = NG > 2 ? 2 : 1;     // a lane's words of each array of the pair's scales and bases
    static_assert(WAVES == 4 || WAVES == 8);
    __shared__ uint4 kf_sh[2][FRAGS][64], vf_sh[2][FRAGS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4;
    // (the last rows see the most positions: their blocks start first)
    const int tile = a.tiles - 1 - int(a.target ? blockIdx.y : blockIdx.x), h = a.target ? blockIdx.x : blockIdx.y;
    const Piece piece = this_piece(a, tile, tile == a.tiles - 1 && h == 0 && threadIdx.x < 64 ? a.err : nullptr);
    if (piece.count == 0) return;
    const Seq &s = piece.s;
    const int G = a.group, rows = s.n * G, row0 = tile * ROWS;
    if (row0 >= rows) return;
    const int2 range = tile_blocks(a, piece, row0, min(row0 + ROWS, rows));
    const int b0 = range.x, b1 = range.y, p_seen = first_seen(s, a.window);
    const uint8_t *seq = a.cache + (size_t(piece.seq) * a.n_kv + h) * (a.batch.max_pos / kPos) * block_bytes(d);

    // What this wave turns: block `mine_b` of the pair, its keys or values, a half of them (eight waves).
    const int mine_b = (wave >> 1) & 1, part = wave >> 2;
    const bool values = wave & 1;
    // (a half of three groups' values is one and a half of them)
    constexpr int GROUPS = SPLIT == 1 ? NG : (NG + 1) / 2, TAUS = SPLIT == 1 ? 2 : 1;
    const int g_first = part * WORDS / 4;
    uint32_t raw[WORDS], ps[4 * GROUPS], pm[4 * GROUPS], lim[4][LIM];  // codes, scales and bases; all the pair's scales and bases
    auto load = [&](int b) __attribute__((always_inline)) {
        // (past the last block: that one again, masked by its position)
        const uint8_t *block = seq + size_t(min(b + mine_b, b1 - 1)) * block_bytes(d);
        const uint8_t *codes = block + (values ? v_codes(d) : k_codes(d));
        if constexpr (WORDS % 4 == 0) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const uint4 u = dev::load16(codes + (part * (WORDS / 4) + i) * 1024 + lane * 16);
                raw[4 * i] = u.x, raw[4 * i + 1] = u.y, raw[4 * i + 2] = u.z, raw[4 * i + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < WORDS / 2; ++i) {
                const uint2 u = *reinterpret_cast<const uint2 *>(codes + code_offset(part * WORDS + 2 * i, lane));
                raw[2 * i] = u.x, raw[2 * i + 1] = u.y;
            }
        }
        if (values) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const uint8_t *at = block + (g_first + g) * 64 + c * 16;
                const uint4 u = dev::load16(at + v_scales(d)), v = dev::load16(at + v_bases(d));
                ps[4 * g] = u.x, ps[4 * g + 1] = u.y, ps[4 * g + 2] = u.z, ps[4 * g + 3] = u.w;
                pm[4 * g] = v.x, pm[4 * g + 1] = v.y, pm[4 * g + 2] = v.z, pm[4 * g + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                pm[g] = *reinterpret_cast<const uint32_t *>(block + k_bases(d) + g * 64 + n * 4);
#pragma unroll
                for (int tau = 0; tau < TAUS; ++tau)
                    ps[TAUS * g + tau] = *reinterpret_cast<const uint16_t *>(block + k_scales(d) + g * 64 + 2 * order_index(16 * (part + tau) + n));
            }
        }
        // Every wave sees all the scales and bases: LIM pairs of values per lane and array (lane = block, word).
#pragma unroll
        for (int l = 0; l < LIM; ++l) {
            const int w = 32 * l + (lane & 31) % (16 * (NG - 2 * l));
            const uint8_t *all = seq + size_t(min(b + (lane >> 5), b1 - 1)) * block_bytes(d) + 4 * w;
            lim[0][l] = *reinterpret_cast<const uint32_t *>(all + k_scales(d));
            lim[1][l] = *reinterpret_cast<const uint32_t *>(all + k_bases(d));
            lim[2][l] = *reinterpret_cast<const uint32_t *>(all + v_scales(d));
            lim[3][l] = *reinterpret_cast<const uint32_t *>(all + v_bases(d));
        }
    };
    int ek[2] = {0, 0}, ev[2] = {0, 0};  // exponents of the two buffers' keys and values
    auto turn = [&](int b, int buf, int most) __attribute__((always_inline)) {  // most: of the values' exponent
        if ((b + 2) * kPos > s.len || b * kPos < p_seen) {
            // Positions that may never have been written (as in kv4_attend_kernel) may hold anything: their scales and
            // bases count as zeros.
            auto unseen = [&](int at) { return at >= s.len || at < p_seen; };
            const int blk = min(b + (lane >> 5), b1 - 1), w = lane & 15;  // word of the group's 16
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int o = 2 * w + e, in_order = 16 * ((o >> 2) & 1) + 4 * (o >> 3) + (o & 3), in_tiles = 16 * e + w;
                const uint32_t drop = ~(0xffffu << (16 * e));
#pragma unroll
                for (int l = 0; l < LIM; ++l) {
                    if (unseen(blk * kPos + in_order)) lim[0][l] &= drop, lim[2][l] &= drop, lim[3][l] &= drop;
                    if (unseen(blk * kPos + in_tiles)) lim[1][l] &= drop;
                }
            }
            if (values) {
                const int own = min(b + mine_b, b1 - 1);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int k = 2 * i + e;
                        if (!unseen(own * kPos + 16 * (k >> 2) + 4 * c + (k & 3))) continue;
#pragma unroll
                        for (int g = 0; g < GROUPS; ++g) {
                            ps[4 * g + i] &= ~(0xffffu << (16 * e));
                            pm[4 * g + i] &= ~(0xffffu << (16 * e));
                        }
                    }
            }
        }
        ek[buf] = held_exponent(lim[1], lim[0]);
        ev[buf] = min(most, held_exponent(lim[3], lim[2]));
        const float fm = ldexpf(1.f, values ? ev[buf] : ek[buf]), fs = fm * 512.f;  // (codes as u 2^-9)
        uint4 *dst = &(values ? vf_sh : kf_sh)[buf][mine_b * 4 * NG + part * WORDS][lane];
        auto turned = [&](uint32_t w, f16x2 s0, f16x2 s1, f16x2 s2, f16x2 s3, f16x2 m0, f16x2 m1, f16x2 m2, f16x2 m3) {
            constexpr _Float16 l = 0x1p15f, q = 0x1p11f;
            const f16x8 u = raw_codes(w) * f16x8{l, l, q, q, l, l, q, q};
            return __builtin_bit_cast(uint4, u * join8(s0, s1, s2, s3) + join8(m0, m1, m2, m3));
        };
        if (values) {
            f16x2 sc[GROUPS][4], ba[GROUPS][4];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[g][i] = pack_f16(low_half(ps[4 * g + i]) * fs, high_half(ps[4 * g + i]) * fs);
                    ba[g][i] = pack_f16(low_half(pm[4 * g + i]) * fm, high_half(pm[4 * g + i]) * fm);
                }
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                if (NG == 3 && SPLIT == 2 && (w & ~1) == 2 && part) {  // (there the second half's next group begins)
                    dst[w * 64] = turned(raw[w], sc[1][0], sc[1][1], sc[1][2], sc[1][3], ba[1][0], ba[1][1], ba[1][2], ba[1][3]);
                    continue;
                }
                constexpr int last_group = GROUPS - 1;
                const int g = min(w / 4, last_group);
                dst[w * 64] = turned(raw[w], sc[g][0], sc[g][1], sc[g][2], sc[g][3], ba[g][0], ba[g][1], ba[g][2], ba[g][3]);
            }
        } else {
#pragma unroll
            for (int tau = 0; tau < TAUS; ++tau) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float sv = low_half(ps[TAUS * g + tau]) * fs, mv = (part + tau ? high_half(pm[g]) : low_half(pm[g])) * fm;
                    const f16x2 sc = pack_f16(sv, sv), ba = pack_f16(mv, mv);
#pragma unroll
                    for (int j = 2 * g; j < 2 * g + 2; ++j) {
                        const int w = tau * 2 * NG + j;
                        dst[w * 64] = turned(raw[w], sc, sc, sc, sc, ba, ba, ba, ba);
                    }
                }
            }
        }
    };

    // The rows: their queries as operands, scaled as in kv4_attend_kernel; a row past the last repeats it.
    const int w_row0 = row0 + wave * 16 * NT;
    auto row_of = [&](int t) { return min(w_row0 + 16 * t + n, rows - 1); };
    f16x8 bq[NT][2 * NG];
    int last[NT];
    float zs[NT];
    {
        uint4 qraw[NT][2 * NG];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = row_of(t), i = row / G;
            const size_t at = size_t(s.t0 + i) * a.q_stride + size_t(h * G + row - i * G) * d + 8 * c;
            last[t] = s.len - s.n + i;
#pragma unroll
            for (int j = 0; j < 2 * NG; ++j)
                qraw[t][j] = dev::load16(reinterpret_cast<const uint8_t *>(static_cast<const uint16_t *>(a.q) + at + 32 * j));
        }
        if (b0 < b1) load(b0);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float x[2 * NG][8], top = 0.f;
#pragma unroll
            for (int j = 0; j < 2 * NG; ++j) {
                const uint32_t w[4] = {qraw[t][j].x, qraw[t][j].y, qraw[t][j].z, qraw[t][j].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[j][2 * e] = low_half(w[e]);
                    x[j][2 * e + 1] = high_half(w[e]);
                    top = fmaxf(top, fmaxf(fabsf(x[j][2 * e]), fabsf(x[j][2 * e + 1])));
                }
            }
            top = max_over_c(top);
            const int e2 = top > 0.f && top < INFINITY ? min(max(14 - ilogbf(top), -88), 148) : 0;
            zs[t] = row_unit(a.scale, -e2);
#pragma unroll
            for (int j = 0; j < 2 * NG; ++j) {
                f16x8 q1[1];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = ldexpf(a.scale < 0.f ? -x[j][e] : x[j][e], e2);
                split<1>(x[j], q1);
                bq[t][j] = q1[0];
            }
        }
    }

    floatx4 acc[NT][4 * NG], sum[NT];  // sum of 2^(15 + ea) P V (dims x rows), sum of 2^15 P (in every element)
    float mx[NT];                      // the row's largest score, without the keys' power of two
    bool far[NT], any_far = false;     // (as in kv4_attend_kernel)
    int ea = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        mx[t] = -INFINITY;
        far[t] = false;
        sum[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4 * NG; ++i) acc[t][i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if (b0 < b1) turn(b0, 0, 100);
    lds_barrier();
    // (the wave's own rows decide which blocks need no mask)
    const int w_first = s.len - s.n + min(w_row0, rows - 1) / G, w_last = s.len - s.n + min(w_row0 + 16 * NT - 1, rows - 1) / G;
    auto step = [&](int b, int buf) __attribute__((always_inline)) {
        const bool more = b + 2 < b1;
        if (more) load(b + 2);
        __builtin_amdgcn_sched_barrier(0);
        float p[NT][16];
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // 16 positions: block u / 2, tile u % 2
            f16x8 kf[2 * NG];
#pragma unroll
            for (int j = 0; j < 2 * NG; ++j) kf[j] = __builtin_bit_cast(f16x8, kf_sh[buf][u * 2 * NG + j][lane]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                floatx4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 2 * NG; ++j) z = mfma(kf[j], bq[t][j], z);
#pragma unroll
                for (int r = 0; r < 4; ++r) p[t][4 * u + r] = z[r];
            }
        }
        const bool full = (b + 2) * kPos - 1 <= w_first && b + 2 <= b1 && (!a.window || b * kPos > w_last - a.window);
        const float unscale = ldexpf(1.f, -ek[buf]);
        const int e_new = ev[buf];
        f16x8 bp[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (!full) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const int at = (b + (k >> 3)) * kPos + 16 * ((k >> 2) & 1) + 4 * c + (k & 3);
                    if (at > last[t] || at >= b1 * kPos || (a.window && at <= last[t] - a.window)) p[t][k] = -INFINITY;
                }
            }
            float top = p[t][0];
#pragma unroll
            for (int k = 1; k < 16; ++k) top = fmaxf(top, p[t][k]);
            top = max_over_c(top);
            const float was = mx[t], now = fmaxf(was, top * unscale);
            const float to = now == -INFINITY ? 0.f : product(now, zs[t]);
            float by = 15.f - to, unit = fminf(fmaxf(zs[t] * unscale, 0x1p-126f), 0x1p126f);
            if (any_far || e_new != ea || __any(now > was)) {
                const float off = product(was, zs[t]);
                float fall = off - to;
                any_far |= __any(is_far(to));
                if (__builtin_expect(any_far, 0)) {
                    if (is_far(to) || far[t]) {
                        fall = fmaf(was - now, zs[t], far[t] ? 0.f : fmaf(-was, zs[t], off));
                        far[t] = true;
                        by = 15.f;
                        unit = zs[t];
                    }
                    const float same = far[t] ? unscale : 1.f, from = far[t] ? now : 0.f;
#pragma unroll
                    for (int k = 0; k < 16; ++k) p[t][k] = fmaf(p[t][k], same, -from);
                }
                const float f = was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fall), fa = ldexpf(f, e_new - ea);
                mx[t] = now;
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[t][r] *= f;
#pragma unroll
                for (int i = 0; i < 4 * NG; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][i][r] *= fa;
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) p[t][k] = __builtin_amdgcn_exp2f(fmaf(p[t][k], unit, by));
#pragma unroll
            for (int u = 0; u < 2; ++u)
                bp[t][u] = join8(pack_f16(p[t][8 * u], p[t][8 * u + 1]), pack_f16(p[t][8 * u + 2], p[t][8 * u + 3]),
                                 pack_f16(p[t][8 * u + 4], p[t][8 * u + 5]), pack_f16(p[t][8 * u + 6], p[t][8 * u + 7]));
        }
        ea = e_new;
        const _Float16 one = 1.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int t = 0; t < NT; ++t) sum[t] = mfma(f16x8{one, one, one, one, one, one, one, one}, bp[t][u], sum[t]);
#pragma unroll
            for (int i = 0; i < 4 * NG; ++i) {
                const f16x8 vf = __builtin_bit_cast(f16x8, vf_sh[buf][u * 4 * NG + i][lane]);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t][i] = mfma(vf, bp[t][u], acc[t][i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) turn(b + 2, buf ^ 1, ea);
        lds_barrier();
    };
#pragma unroll 1
    for (int b = b0; b < b1; b += 4) {
        step(b, 0);
        if (b + 2 < b1) step(b + 2, 1);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = w_row0 + 16 * t + n;
        if (row >= rows) continue;
        if (piece.count > 1) {
            float *o = a.part + ((size_t(piece.first + piece.split) * a.n_kv + h) * a.tiles * ROWS + row) * (d + 4);
            // (relative to the largest score itself; every piece has the 2^15)
            const float rel = far[t] || mx[t] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(fmaf(-mx[t], zs[t], product(mx[t], zs[t])));
#pragma unroll
            for (int i = 0; i < 4 * NG; ++i)
                *reinterpret_cast<float4 *>(o + 16 * i + 4 * c) =
                    make_float4(ldexpf(acc[t][i][0] * rel, -ea), ldexpf(acc[t][i][1] * rel, -ea), ldexpf(acc[t][i][2] * rel, -ea),
                                ldexpf(acc[t][i][3] * rel, -ea));
            if (c == 0) *reinterpret_cast<float4 *>(o + d) = make_float4(mx[t], sum[t][0] * rel, zs[t], 0.f);
            continue;
        }
        const float l = sum[t][0], inv = l == 0.f ? 0.f : 1.f / l;
        const size_t at = size_t(s.t0 + row / G) * a.out_stride + size_t(h * G + row % G) * d + 4 * c;
#pragma unroll
        for (int i = 0; i < 4 * NG; ++i)
            store4<false>(a.out, at + 16 * i, make_float4(ldexpf(acc[t][i][0] * inv, -ea), ldexpf(acc[t][i][1] * inv, -ea),
                                                          ldexpf(acc[t][i][2] * inv, -ea), ldexpf(acc[t][i][3] * inv, -ea)));
    }
}

// One more piece (its maximum, sum and the row's unit; four dims of its output).  As in the attention kernel: nothing
// seen counts 0, NaN stays.
__device__ __forceinline__ void join_piece(float &M, float &S, float4 &v, float4 ml, float4 u) {
    const float now = fmaxf(M, ml.x);
    const float f = M == -INFINITY && S == 0.f ? 0.f : __builtin_amdgcn_exp2f((M - now) * ml.z);
    const float g = ml.x == -INFINITY && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((ml.x - now) * ml.z);
    M = now;
    S = fmaf(S, f, ml.y * g);
    v.x = fmaf(v.x, f, u.x * g);
    v.y = fmaf(v.y, f, u.y * g);
    v.z = fmaf(v.z, f, u.z * g);
    v.w = fmaf(v.w, f, u.w * g);
}

// Joins the pieces of one row.  grid: (rows, key/value head, sequence); groups of d / 4 lanes take the pieces in
// turn, a running maximum each.
template <int NG, bool F32>
__global__ __launch_bounds__(kAttBlock) void kv4_join_kernel(AttendArgs a, int tile_rows) {
    constexpr int d = NG * kGroup, N4 = d / 4, SUB = kAttBlock / N4;
    __shared__ float4 acc_sh[SUB][N4];
    __shared__ float max_sh[SUB], sum_sh[SUB];
    const Piece piece = find_piece(a, blockIdx.z, false, nullptr);
    if (piece.count <= 1) return;
    const Seq &s = piece.s;
    const int G = a.group, row = blockIdx.x, h = blockIdx.y;
    if (row >= s.n * G) return;
    const int tid = threadIdx.x, i4 = tid % N4, sub = tid / N4;
    const size_t step = size_t(a.n_kv) * a.tiles * tile_rows * (d + 4);
    const float *p = a.part + ((size_t(piece.first) * a.n_kv + h) * a.tiles * tile_rows + row) * (d + 4);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float M = -INFINITY, S = 0.f, unit = 0.f;  // (the group that ends the work has the first piece)
    if (sub < SUB) {
#pragma unroll 4
        for (int k = sub; k < piece.count; k += SUB) {
            const float4 ml = *reinterpret_cast<const float4 *>(p + k * step + d);
            const float4 u = *reinterpret_cast<const float4 *>(p + k * step + 4 * i4);
            join_piece(M, S, v, ml, u);
            unit = ml.z;
        }
        acc_sh[sub][i4] = v;
        if (i4 == 0) {
            max_sh[sub] = M;
            sum_sh[sub] = S;
        }
    }
    __syncthreads();
    if (tid >= N4) return;
    float top = max_sh[0];
#pragma unroll
    for (int k = 1; k < SUB; ++k) top = fmaxf(top, max_sh[k]);
    S = 0.f;
    v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < SUB; ++k) {
        const float f = max_sh[k] == -INFINITY && sum_sh[k] == 0.f ? 0.f : __builtin_amdgcn_exp2f((max_sh[k] - top) * unit);
        const float4 u = acc_sh[k][tid];
        S = fmaf(f, sum_sh[k], S);
        v.x = fmaf(f, u.x, v.x);
        v.y = fmaf(f, u.y, v.y);
        v.z = fmaf(f, u.z, v.z);
        v.w = fmaf(f, u.w, v.w);
    }
    const float inv = S == 0.f ? 0.f : 1.f / S;
    v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
    store4<F32>(a.out, size_t(s.t0 + row / G) * a.out_stride + size_t(h * G + row % G) * d + 4 * tid, v);
}

// The same for many rows: a group of d / 4 lanes takes one row and its pieces one after the other.  grid: (groups of
// rows, key/value head, sequence)
template <int NG, bool F32>
__global__ __launch_bounds__(kAttBlock) void kv4_join_rows_kernel(AttendArgs a, int tile_rows) {
    constexpr int d = NG * kGroup, N4 = d / 4, ROWS = kAttBlock / N4;
    const Piece piece = find_piece(a, blockIdx.z, false, nullptr);
    if (piece.count <= 1) return;
    const Seq &s = piece.s;
    const int G = a.group, i4 = threadIdx.x % N4, sub = threadIdx.x / N4, row = blockIdx.x * ROWS + sub, h = blockIdx.y;
    if (sub >= ROWS || row >= s.n * G) return;
    const size_t step = size_t(a.n_kv) * a.tiles * tile_rows * (d + 4);
    const float *p = a.part + ((size_t(piece.first) * a.n_kv + h) * a.tiles * tile_rows + row) * (d + 4);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float M = -INFINITY, S = 0.f;
#pragma unroll 4
    for (int k = 0; k < piece.count; ++k) {
        const float4 ml = *reinterpret_cast<const float4 *>(p + k * step + d);
        join_piece(M, S, v, ml, *reinterpret_cast<const float4 *>(p + k * step + 4 * i4));
    }
    const float inv = S == 0.f ? 0.f : 1.f / S;
    v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
    store4<F32>(a.out, size_t(s.t0 + row / G) * a.out_stride + size_t(h * G + row % G) * d + 4 * i4, v);
}

// What a call launches: from its sizes alone, since lengths are on the device (max_pos bounds them).
struct AttendPlan {
    int prompt;     // waves of the kernel for many rows, or 0
    int tiles;      // otherwise: tiles of 16 rows per wave (0: one of 8)
    int tile_rows, blocks;  // rows per block, blocks of the largest sequence's rows
    int target, least, units;
    size_t workspace;
};
AttendPlan attend_plan(int n_seq, int n_kv, int group, int d, int max_q, int max_pos, bool f32) {
    const long long rows = (long long)max_q * group;
    AttendPlan p{};
    int fill = kTarget;
    // Many rows: keys and values turned to fp16 once for a block's rows.  It starts later and goes on faster: with 32
    // query and 4 key/value heads of 128, 128 tokens over 1024 positions take 21.9 us (the other kernel 27.1), 300 over
    // 8000 79.5 (226), 2048 over 8192 329 (865); with 16 heads of 256, 300 over 8000 81 (253); with 32 of 64, 64 over
    // 4000 19.4 (29.4).  Where the rule begins the other kernel is still ahead: 64 over 512 19.5 (14.7), 32 over 1024
    // 19.9 (15.2).
    if (!f32 && rows >= 128 && double(rows) * n_kv * n_seq * max_pos * d >= double(1 << 27)) {
        const int per = 64 * prompt_tiles(d);  // rows of four waves
        const long long four = (rows + per - 1) / per * n_kv * n_seq, eight = (rows + 2 * per - 1) / (2 * per) * n_kv * n_seq;
        // Eight waves turn half as often as two blocks of four: taken where they fill the device (2048 tokens over
        // 8192 positions: 329 us, four 362), and for heads of more than 128, of which a unit holds one block, where the
        // positions are split (300 tokens, 16 heads of 256, 8000 positions: 81 us, four 140).
        fill = d <= 128 ? 512 : 256;
        // Longer pieces where rows and heads already give a quarter of the blocks: they keep short caches whole (296 tokens
        // of 3 sequences, 32 heads of 128, up to 325 positions: 20 us, 31 with 8; 370, 64 heads, 593 positions: 23 and 28).
        // Where the positions are more, or heads are larger, 8 would be faster (600 tokens, 32 heads of 64, 1000 positions:
        // 25.0 us, 23.7 with 8; 611 of 4 sequences, 4 heads of 192, 751 positions: 37.6 and 29.4); below a quarter 16 would
        // be slower (128 tokens, 32 heads of 128, 2000 positions: 23.7 us, 29.8 with 16).
        p.least = four * 4 >= fill ? 16 : 8;
        p.prompt = eight >= 256 || (d > 128 && rows > per && four * 3 <= fill * 2) ? 8 : 4;
        p.tile_rows = per * (p.prompt / 4);
        if (p.prompt == 8) fill = 256;
    } else {
        const int most = d <= 64 ? (f32 ? 2 : 4) : d <= 128 ? 2 : d <= 192 && !f32 ? 2 : 1;  // what a wave's registers hold
        p.tiles = rows <= 8 ? 0 : rows <= 16 ? 1 : rows <= 32 ? std::min(2, most) : most;
        p.tile_rows = p.tiles ? 16 * p.tiles : 8;
        p.least = kAttWaves;
    }
    p.blocks = int((rows + p.tile_rows - 1) / p.tile_rows);
    const long long base = (long long)p.blocks * n_kv;  // blocks per sequence or piece
    const long long pieces = (max_pos / kPos + p.least - 1) / p.least;  // most that a sequence has
    // Split where that makes more blocks; many rows, whose pieces' outputs cost more, where it makes twice as many (300
    // tokens, 32 heads of 128, 8000 positions: 258 us whole, 79 split; 1556 rows of 4 heads of 64 in each of 6 sequences
    // of up to 701, 312 blocks: 24 whole, 31 split).  (By the number of blocks alone: a batch that fills the device by it is
    // not split, however unequal its sequences are.)
    if ((p.prompt ? base * n_seq * 2 <= fill : base * n_seq < fill) && pieces > 1) {
        p.target = int(std::min(std::max(1ll, fill / base), pieces * n_seq));
        p.units = p.target + n_seq - 1;  // (rounding up leaves less than one piece more per sequence)
        p.workspace = (size_t(p.units) * n_kv * p.blocks * p.tile_rows * (d + 4) * sizeof(float) + 255) & ~size_t(255);
    }
    return p;
}

}  // namespace

size_t kv4_attention_workspace_bytes(int, int n_seq, int n_heads, int n_kv, int d, int max_q, int max_pos) {
    return std::max(attend_plan(n_seq, n_kv, n_heads / n_kv, d, max_q, max_pos, false).workspace,
                    attend_plan(n_seq, n_kv, n_heads / n_kv, d, max_q, max_pos, true).workspace);
}

hipError_t launch_kv4_attention(const void *q, int dtype, long long q_stride, const void *cache, const kv4::Batch &batch,
                                int n_heads, int n_kv, int d, int window, float scale, void *out, long long out_stride,
                                void *workspace, int *err, hipStream_t s) {
    const bool f32 = dtype == MOE_F32;
    const AttendPlan p = attend_plan(batch.n_seq, n_kv, n_heads / n_kv, d, batch.max_q, batch.max_pos, f32);
    AttendArgs a;
    a.q = q;
    a.out = out;
    a.cache = static_cast<const uint8_t *>(cache);
    a.part = static_cast<float *>(workspace);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.n_heads = n_heads;
    a.n_kv = n_kv;
    a.group = n_heads / n_kv;
    a.window = window;
    a.target = p.target;
    a.least = p.least;
    a.unit = p.prompt ? 2 : 1;
    a.tiles = p.blocks;
    a.scale = scale * 1.44269504088896341f;
    a.batch = batch;
    a.err = err;
    const dim3 grid = p.target ? dim3(n_kv, p.blocks, p.units) : dim3(p.blocks, n_kv, batch.n_seq);
    if (p.prompt) {
#define KV4_PROMPT(NG, W) \
    if (d == NG * kGroup && p.prompt == W) kv4_prompt_kernel<NG, W><<<grid, 64 * W, 0, s>>>(a);
        KV4_PROMPT(1, 4) KV4_PROMPT(1, 8) KV4_PROMPT(2, 4) KV4_PROMPT(2, 8) KV4_PROMPT(3, 4) KV4_PROMPT(3, 8) KV4_PROMPT(4, 4) KV4_PROMPT(4, 8)
#undef KV4_PROMPT
    } else {
#define KV4_RUN(NG, NT, F) kv4_attend_kernel<NG, NT ? NT : 1, F, NT == 0><<<grid, kAttBlock, 0, s>>>(a)
#define KV4_CASE(NG, NT, F) case (NG * 2 + F) * 8 + NT: KV4_RUN(NG, NT, F); break;
    switch ((d / kGroup * 2 + f32) * 8 + p.tiles) {
        KV4_CASE(1, 0, false) KV4_CASE(1, 1, false) KV4_CASE(1, 2, false) KV4_CASE(1, 4, false)
        KV4_CASE(1, 0, true) KV4_CASE(1, 1, true) KV4_CASE(1, 2, true)
        KV4_CASE(2, 0, false) KV4_CASE(2, 1, false) KV4_CASE(2, 2, false)
        KV4_CASE(2, 0, true) KV4_CASE(2, 1, true) KV4_CASE(2, 2, true)
        KV4_CASE(3, 0, false) KV4_CASE(3, 1, false) KV4_CASE(3, 2, false)
        KV4_CASE(3, 0, true) KV4_CASE(3, 1, true)
        KV4_CASE(4, 0, false) KV4_CASE(4, 1, false)
        KV4_CASE(4, 0, true) KV4_CASE(4, 1, true)
    default: return hipErrorInvalidValue;
    }
#undef KV4_CASE
#undef KV4_RUN
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.target) return e;
    const int rows = batch.max_q * a.group;
    // One block per row has its pieces in flight together, a group of lanes per row needs fewer blocks: 64 tokens, 32 heads
    // of 64, 4000 positions (2048 rows) 19.3 and 19.4 us with the attention, 128 (4096 rows) 26.1 and 22.7.
    const bool many = (long long)rows * n_kv * batch.n_seq >= 2048;
#define KV4_JOIN(NG, F)                                                                                             \
    if (d == NG * kGroup && f32 == F) {                                                                             \
        constexpr int per = kAttBlock / (NG * kGroup / 4);                                                          \
        if (many) kv4_join_rows_kernel<NG, F><<<dim3((rows + per - 1) / per, n_kv, batch.n_seq), kAttBlock, 0, s>>>(a, p.tile_rows); \
        else kv4_join_kernel<NG, F><<<dim3(rows, n_kv, batch.n_seq), kAttBlock, 0, s>>>(a, p.tile_rows);            \
    }
    KV4_JOIN(1, false) KV4_JOIN(1, true) KV4_JOIN(2, false) KV4_JOIN(2, true)
    KV4_JOIN(3, false) KV4_JOIN(3, true) KV4_JOIN(4, false) KV4_JOIN(4, true)
#undef KV4_JOIN
    return hipGetLastError();
}

}  // namespace moe
