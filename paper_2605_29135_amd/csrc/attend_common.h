// attend_common.h -- what the attention kernels over a cache of a batch share: operands and lane moves of the 16x16x32
// matrix product (lane l: row or column n = l % 16, elements 8 c + i, c = l / 16), and the split of a ragged batch over
// blocks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "kv4.h"

namespace moe {
namespace attend {

using kv4::Batch;
using kv4::Seq;
using kv4::sequence;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma(f16x8 a, f16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // round to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {__bf16(lo), __bf16(hi)};
    return __builtin_bit_cast(uint32_t, v);
}

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

// The split of a batch: sequences are cut into pieces of `chunk` blocks of positions, at least `least`, so
// that there are about `target` of them in all; a sequence has at least one piece.  Every wave works it out for
// itself.  by_unit: which piece is number `want`; otherwise, the pieces of sequence `want`.
struct Piece {
    Seq s;
    int seq, split, chunk;
    int first, count;  // of the sequence's pieces (count 0: there is no such piece)
};
// blocks(sequence): the blocks of positions that its tokens see.
struct Split {
    int target;  // pieces of a whole batch (0: every sequence in one piece)
    int least;   // blocks of positions that a piece has at least; the rest come in multiples of `unit`
    int unit;
};
template <typename F>
__device__ __forceinline__ Piece find_piece(const Batch &b, const Split &split, F blocks, int want, bool by_unit, int *err) {
    const int target = split.target;
    const int lane = threadIdx.x & 63;
    uint32_t total = 0;  // (a batch that is split has fewer than kTarget sequences of at most 2^21 blocks)
    Seq s{0, 0, 0, false};
    int nb = 0;
    auto look = [&](int base) {
        s = Seq{0, 0, 0, false};
        if (base + lane < b.n_seq) s = sequence(b, base + lane);
        nb = blocks(s);
    };
#pragma unroll 1
    for (int base = 0; base < b.n_seq; base += 64) {
        look(base);
        if (err && s.bad) atomicOr(err, kErrRange);
        total += uint32_t(__builtin_amdgcn_readlane(int(wave_scan(uint32_t(nb))), 63));
    }
    Piece p{};
    p.chunk = max(int((total + uint32_t(target) - 1) / uint32_t(target)), split.least);
    p.chunk = (p.chunk + split.unit - 1) & -split.unit;
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
            chunk = (p.chunk + p.chunk * k / 8 + split.unit - 1) & -split.unit;
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

template <bool F32>
__device__ __forceinline__ void store4(void *out, size_t at, float4 v) {
    if constexpr (F32) *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = v;
    else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// A barrier for what the block's waves pass one another through LDS; loads in flight stay so.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// One more piece (its maximum, sum and the row's unit; four dims of its output).  A piece that saw nothing (the
// maximum -inf, the sum 0) counts 0, NaN stays.
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

// Joining: Args has part ([unit][head][tiles][tile_rows][d + 4]: a row's unnormalised output, maximum, sum and unit, which
// takes differences of maxima to log2), out, out_stride, group, n_kv and tiles, and split_piece(args, want, by_unit, err)
// finds a sequence's pieces.
constexpr int kJoinBlock = 256;

// Joins the pieces of one row.  grid: (rows, key/value head, sequence); groups of d / 4 lanes take the pieces in
// turn, a running maximum each.
template <int NG, bool F32, typename Args>
__global__ __launch_bounds__(kJoinBlock) void join_kernel(Args a, int tile_rows) {
    constexpr int d = NG * 64, N4 = d / 4, SUB = kJoinBlock / N4;
    __shared__ float4 acc_sh[SUB][N4];
    __shared__ float max_sh[SUB], sum_sh[SUB];
    const Piece piece = split_piece(a, blockIdx.z, false, nullptr);
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
template <int NG, bool F32, typename Args>
__global__ __launch_bounds__(kJoinBlock) void join_rows_kernel(Args a, int tile_rows) {
    constexpr int d = NG * 64, N4 = d / 4, ROWS = kJoinBlock / N4;
    const Piece piece = split_piece(a, blockIdx.z, false, nullptr);
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

// Joins rows (of the largest sequence) of n_seq sequences.
template <int NG, bool F32, typename Args>
void launch_join(const Args &a, int rows, int n_seq, int tile_rows, hipStream_t s) {
    // One block per row has its pieces in flight together, a group of lanes per row needs fewer blocks: 64 tokens, 32 heads
    // of 64, 4000 positions (2048 rows) 19.3 and 19.4 us with the attention over the 4-bit cache, 128 (4096 rows) 26.1 and
    // 22.7.
    constexpr int per = kJoinBlock / (NG * 64 / 4);
    if ((long long)rows * a.n_kv * n_seq >= 2048)
        join_rows_kernel<NG, F32><<<dim3((rows + per - 1) / per, a.n_kv, n_seq), kJoinBlock, 0, s>>>(a, tile_rows);
    else
        join_kernel<NG, F32><<<dim3(rows, a.n_kv, n_seq), kJoinBlock, 0, s>>>(a, tile_rows);
}

}  // namespace attend
}  // namespace moe
