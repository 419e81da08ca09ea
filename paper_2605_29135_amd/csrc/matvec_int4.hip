// matvec_int4.hip -- matrix-vector products with int4-g128 weights for 1 to 16 tokens.
//
// y[t] = add[t] + W h[t].  The bound is the weights' bytes.  On the matrix cores a 16-row tile of W is an operand
// as it lies in memory (lane l: row l % 16, 16 bytes = 32 columns of the quantisation group, quarter l / 16), so
// the work per weight does not depend on the number of tokens.  The codes enter as fp16 q 2^-9 (a nibble with its
// top bit flipped is the subnormal (q + 8) 2^-24, which a packed fma takes there), the tokens' values, scaled by a
// power of two per token and wave so that the largest is in [2^14, 2^15), as two fp16 terms (2^-22 of that largest
// value); every product is exact, and the group's scale multiplies its fp32 sum.  Up to 8 tokens the two terms
// are rows of one product; for more they are two products.
//
// A block takes items of RB row tiles; its eight waves share the columns.  With few tokens a wave forms the terms of its
// columns once (lanes over columns), turns them into operands through its own part of LDS and keeps those in registers
// from item to item; with more a launch of its own forms every token's, which the blocks read.  A tile's next weights are
// loaded as soon as it has been multiplied.  Many rows: see matvec_stream_kernel.
//
// Measured: 5120 x 2048, 1 token 5.5 us (5.4 MB, 1 TB/s: a launch, the chain of loads and the sum over waves); 2048 x
// 4096, 16 tokens 3.4 us for the terms and 6.6 us (half of the units have a block); 131071 x 2048, 3 tokens 32.8 us
// (140 MB, 4.3 TB/s; weights that change from pass to pass).
#include "device_common.h"
#include "internal.h"

#include <type_traits>

namespace moe {
namespace {

using dev::kWave;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kMvWaves = 8, kMvBlock = kMvWaves * kWave;
constexpr int kMvGrid = 256;  // compute units
constexpr int kMvFit = 2 * kMvGrid;  // blocks that run together
// Tokens whose terms every block forms itself: 5120 x 4096 with 3 tokens takes 9.4 us, with 4 and a launch for them 11.1;
// 9 tokens took 24.6 us without that launch and 15.7 with it.
constexpr int kMvTokens = 3;
constexpr int kCodeExp = -9;
constexpr int kTermsBlock = 1024;

// The eight codes of a dword as fp16 q 2^-9, in the order 0,4,1,5,2,6,3,7.  (Nibbles at bits 4-7 of a half are 16
// times those at 0-3, which their factor takes back.)
__device__ __forceinline__ f16x8 codes(uint32_t w) {
    constexpr uint32_t L = 0x000F000Fu, H = 0x00F000F0u;
    constexpr _Float16 m = 0x1p15f, n = 0x1p11f, a = -0x1p-6f;
    const uint32_t v = w ^ 0x88888888u, u = v >> 8;
    return __builtin_bit_cast(f16x8, make_uint4(v & L, v & H, u & L, u & H)) * f16x8{m, m, n, n, m, m, n, n} +
           f16x8{a, a, a, a, a, a, a, a};
}

// One output in fp32, element by element: what a sum that is not finite is taken from (an infinite value has no
// terms, or a sum overflows where the definition's does not).
__device__ float row_dot(const uint8_t *w, const uint16_t *scale, const float *x, float inv, int K) {
    float acc = 0.f;
#pragma unroll 1
    for (int g = 0; g < K / 128; ++g) {
        const float s = dev::bf16_bits_to_float(scale[g]);
        float part = 0.f;
#pragma unroll 1
        for (int i = 0; i < 128; ++i) {
            const int q = int(__builtin_amdgcn_sbfe(uint32_t(w[g * 64 + i / 2]), 4 * (i & 1), 4));
            part = fmaf(s * float(q), x[g * 128 + i] * inv, part);  // (s q is exact)
        }
        acc += part;
    }
    return acc;
}

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

__device__ __forceinline__ float squares_of(float4 u) { return fmaf(u.x, u.x, fmaf(u.y, u.y, fmaf(u.z, u.z, u.w * u.w))); }

// 1 / sqrt(mean x^2 + 1e-6) from the sum of squares, or, where that is past the largest number, from the squares of
// x 2^-100 (one lane, a group at a time; an infinite x leaves 0, a NaN stays).
__device__ float norm_factor(float squares, const float *x, int K) {
    if (finite(squares)) return rsqrtf(squares / float(K) + 1e-6f);
    squares = 0.f;
#pragma unroll 1
    for (int g = 0; g < K / 128; ++g) {
        float part = 0.f;
#pragma unroll 4
        for (int i = 0; i < 32; ++i) {
            const float4 u = dev::load_f4(reinterpret_cast<const float4 *>(x) + g * 32 + i);
            part += squares_of(make_float4(u.x * 0x1p-100f, u.y * 0x1p-100f, u.z * 0x1p-100f, u.w * 0x1p-100f));
        }
        squares += part;
    }
    return rsqrtf(squares / float(K)) * 0x1p-100f;
}

// Largest magnitude over the wave, in every lane.
__device__ __forceinline__ float wave_top(float v) {
    v = fmaxf(v, dev::dpp<0xB1>(v));
    v = fmaxf(v, dev::dpp<0x4E>(v));
    v = fmaxf(v, dev::dpp<0x141>(v));
    v = fmaxf(v, dev::dpp<0x140>(v));
    auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
    return fmaxf(fmaxf(lane(0), lane(16)), fmaxf(lane(32), lane(48)));
}
// A barrier for what the block's waves pass one another through LDS.  (__syncthreads would also wait for the weights
// in flight.)
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ uint32_t bits(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// Four neighbouring columns of a token, scaled by 2^e2, as two fp16 terms in the operands' order.  Two neighbouring
// lanes hold a dword's eight columns and trade halves, so that each stores two pairs (columns e and e + 4):
// operand(term) is the dword's 16 bytes of that term.
template <typename F>
__device__ __forceinline__ void store_terms(float4 u, int e2, bool odd, F operand) {
    const float a[4] = {ldexpf(u.x, e2), ldexpf(u.y, e2), ldexpf(u.z, e2), ldexpf(u.w, e2)};
    f16x2 h[2] = {f16x2{_Float16(a[0]), _Float16(a[1])}, f16x2{_Float16(a[2]), _Float16(a[3])}};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t got = uint32_t(__builtin_amdgcn_update_dpp(0, int(odd ? bits(h[0]) : bits(h[1])), 0xB1, 0xF, 0xF, false));
        const uint32_t lo = odd ? got : bits(h[0]), hi = odd ? bits(h[1]) : got;  // columns e, e + 1 and e + 4, e + 5
        reinterpret_cast<uint2 *>(operand(k))[odd] =
            make_uint2(__builtin_amdgcn_perm(hi, lo, 0x05040100u), __builtin_amdgcn_perm(hi, lo, 0x07060302u));
        if (k == 0)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                h[e] = f16x2{_Float16(a[2 * e] - float(h[e][0])), _Float16(a[2 * e + 1] - float(h[e][1]))};
    }
}
__device__ __forceinline__ float top_of(float4 u) {
    return fmaxf(fmaxf(fabsf(u.x), fabsf(u.y)), fmaxf(fabsf(u.z), fabsf(u.w)));
}
__device__ __forceinline__ int exponent_of(float top) { return top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 0; }

// Bytes of LDS: the waves' operands (2 T rows: the two terms of each token), then their partial sums.
__host__ __device__ constexpr int stage_bytes(int T, int GS) { return kMvWaves * GS * 512 * T; }
__host__ __device__ constexpr int lds_bytes(int T, int GS, int RB) { return stage_bytes(T, GS) + kMvWaves * RB * 4 * kWave * 4; }

// The terms of every token, once for all the blocks of a call: one block per token (16 of 4096 columns 3.4 us, which is a
// launch and its chain of loads, two reductions and stores).  ws: what takes the sums back (int
// [16]), the norms' factors (float [16]), then at 256 bytes the operands [K / 32][4][2 T rows].
struct Terms {
    const int *back;
    const float *inv;
    const uint4 *operands;
};
__host__ __device__ inline Terms terms_in(const void *ws) {
    const auto *p = static_cast<const uint8_t *>(ws);
    return {reinterpret_cast<const int *>(p), reinterpret_cast<const float *>(p + 64), reinterpret_cast<const uint4 *>(p + 256)};
}
__global__ __launch_bounds__(kTermsBlock) void matvec_terms_kernel(const float *__restrict__ x, int T, int K, bool norm, uint8_t *ws) {
    constexpr int WAVES = kTermsBlock / kWave;
    __shared__ float tops[WAVES], sums[WAVES];
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float4 *xr = reinterpret_cast<const float4 *>(x + size_t(t) * K);
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    float4 held[2];  // (8192 columns; the rest is read again)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int i = tid + u * kTermsBlock;
        held[u] = i < K / 4 ? dev::load_f4(xr + i) : zero;
    }
    float top = fmaxf(top_of(held[0]), top_of(held[1])), squares = squares_of(held[0]) + squares_of(held[1]);
#pragma unroll 1
    for (int i = tid + 2 * kTermsBlock; i < K / 4; i += kTermsBlock) {
        const float4 u = dev::load_f4(xr + i);
        top = fmaxf(top, top_of(u));
        squares += squares_of(u);
    }
    top = wave_top(top);
    squares = dev::wave_sum(squares);
    if (lane == 0) tops[wave] = top, sums[wave] = squares;
    __syncthreads();
    top = tops[0], squares = sums[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w]), squares += sums[w];
    const int e2 = exponent_of(top);
    if (tid == 0) {
        reinterpret_cast<int *>(ws)[t] = -kCodeExp - e2;
        reinterpret_cast<float *>(ws + 64)[t] = norm ? norm_factor(squares, x + size_t(t) * K, K) : 1.f;
    }
    uint4 *out = reinterpret_cast<uint4 *>(ws + 256) + t;
    auto store = [&](int i, float4 u) {  // (K / 4 is a multiple of 32: a pair of lanes stays together)
        uint4 *f = out + size_t((i >> 5) * 16 + ((i >> 1) & 3) * 4 + ((i >> 3) & 3)) * (2 * T);
        store_terms(u, e2, lane & 1, [&](int k) { return f + k * T; });
    };
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (tid + u * kTermsBlock < K / 4) store(tid + u * kTermsBlock, held[u]);
#pragma unroll 1
    for (int i = tid + 2 * kTermsBlock; i < K / 4; i += kTermsBlock) store(i, dev::load_f4(xr + i));
}

// GS: quantisation groups per wave and pass over the columns; MULTI: several passes, the terms formed again for
// each.  LOOP: a block has more than one item or pass.  ONE: the two terms share one product (T <= 8).  PRE: the terms
// come from matvec_terms_kernel (else T <= kMvTokens).
template <int RB, int GS, bool ONE, bool MULTI, bool LOOP, bool PRE>
__global__ __launch_bounds__(kMvBlock, 2) void matvec_int4_kernel(const float *__restrict__ x, const uint8_t *__restrict__ w,
                                                                  int T, int N, int K, const float *add, float *y, bool norm,
                                                                  int items, const void *ws) {
    static_assert(PRE || ONE, "");
    constexpr int NP = ONE ? 1 : 2;  // products
    extern __shared__ uint4 lds[];
    __shared__ float sq[kMvWaves][kMvTokens];  // sums of squares
    __shared__ int exps[kMvWaves][kMvTokens];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, n = lane & 15, c = lane >> 4;
    const int KG = K / 128, passes = MULTI ? (KG + kMvWaves * GS - 1) / (kMvWaves * GS) : 1;
    const int share = (KG + kMvWaves * passes - 1) / (kMvWaves * passes);  // groups per wave and pass, <= GS
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(w + size_t(N) * (K / 2));
    uint4 *stage = lds + wave * (GS * 32 * T);
    float *red = reinterpret_cast<float *>(lds) + (PRE ? 0 : stage_bytes(T, GS) / 4);
    const Terms pre = terms_in(ws);

    struct Weights {
        uint4 w[GS][RB];
        uint32_t sc[GS][RB];
    } b0, b1;
    auto load_tile = [&](Weights &b, int item, int pass, int j) __attribute__((always_inline)) {
        const size_t row = min((item * RB + j) * 16 + n, N - 1);
#pragma unroll
        for (int r = 0; r < GS; ++r) {
            const int g = min((pass * kMvWaves + wave) * share + min(r, share - 1), KG - 1);  // (past the end: not used)
            b.w[r][j] = dev::load16(w + row * (K / 2) + size_t(g) * 64 + 16 * c);
            b.sc[r][j] = scales[row * KG + g];
        }
    };
    f16x8 xt[GS][4][NP];
    int back[4];  // what takes the sums of row 4 c + q of the product back
    // The wave's columns of every token: four per lane and step of 256, scaled, in two terms.
    auto convert = [&](int pass, bool measure) __attribute__((always_inline)) {
        if constexpr (PRE) {
#pragma unroll
            for (int r = 0; r < GS; ++r) {
                const int g = min((pass * kMvWaves + wave) * share + min(r, share - 1), KG - 1);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < NP; ++k)
                        xt[r][j][k] = __builtin_bit_cast(f16x8, pre.operands[size_t((g * 4 + j) * 4 + c) * (2 * T) +
                                                                             (ONE ? min(n, 2 * T - 1) : k * T + min(n, T - 1))]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = 4 * c + q, t = ONE && row >= T ? row - T : row;
                back[q] = pre.back[min(t, T - 1)];
            }
            return;
        }
        const int g0 = (pass * kMvWaves + wave) * share, odd = lane & 1;
        float4 v[kMvTokens][GS / 2];  // (all their loads in flight together)
#pragma unroll
        for (int t = 0; t < kMvTokens; ++t)
#pragma unroll
            for (int i = 0; i < GS / 2; ++i) {
                const int r = 2 * i + (lane >> 5), g = g0 + r;
                v[t][i] = dev::load_f4(reinterpret_cast<const float4 *>(x + size_t(min(t, T - 1)) * K +
                                                                        min(g, KG - 1) * 128 + 4 * (lane & 31)));
                if (r >= share || g >= KG) v[t][i] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
        for (int t = 0; t < kMvTokens; ++t) {
            if (t >= T) break;
            float top = 0.f, squares = 0.f;
#pragma unroll
            for (int i = 0; i < GS / 2; ++i) {
                top = fmaxf(top, top_of(v[t][i]));
                squares += squares_of(v[t][i]);
            }
            top = wave_top(top);
            const int e2 = exponent_of(top);
            if (lane == 0) exps[wave][t] = e2;
            if (norm && measure) {
                squares = dev::wave_sum(squares);
                if (lane == 0) sq[wave][t] = pass ? sq[wave][t] + squares : squares;
            }
#pragma unroll
            for (int i = 0; i < GS / 2; ++i) {
                const int j = (lane >> 1) & 3, part = (lane >> 3) & 3, r = 2 * i + (lane >> 5);
                uint4 *f = stage + ((r * 4 + j) * 4 + part) * (2 * T) + t;
                store_terms(v[t][i], e2, odd, [&](int k) { return f + k * T; });
            }
        }
        // the operands are this wave's own: a wave-level LDS sync
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        // (rows past the last token repeat it and are not stored)
#pragma unroll
        for (int r = 0; r < GS; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < NP; ++k)
                    xt[r][j][k] = __builtin_bit_cast(f16x8, stage[((r * 4 + j) * 4 + c) * (2 * T) + (ONE ? min(n, 2 * T - 1) : k * T + min(n, T - 1))]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int row = 4 * c + q, t = ONE && row >= T ? row - T : row;
            back[q] = -kCodeExp - exps[wave][min(t, T - 1)];
        }
    };

    const int first = blockIdx.x;
#pragma unroll
    for (int j = 0; j < RB; ++j) load_tile(b0, first, 0, j);
    convert(0, true);
    // Output o = tid of the item: row o % (16 RB), token o / (16 RB) (16 RB T <= 512 of them).
    const int o_row = tid % (16 * RB), o_token = tid / (16 * RB);
    int item = first, pass = 0;
    floatx4 sum[RB];
    float addend = 0.f;
    // One pass over one item; `more`: the weights of the next one are loaded meanwhile (past the last: some again, not
    // used).
    auto unit = [&](const Weights &b, Weights &next, auto more) __attribute__((always_inline)) {
        const bool last = pass == passes - 1;
        const int item_next = last ? item + int(gridDim.x) : item, pass_next = last ? 0 : pass + 1;
        const int row = item * 16 * RB + o_row;
        const bool mine = o_token < T && row < N;
        const size_t at = mine ? size_t(o_token) * N + row : 0;
        if (MULTI && (pass || item != first)) convert(pass, item == first);
        // (the addend ahead of the next weights, whose arrival a later load would wait for)
        if (add && last) addend = add[at];
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            if constexpr (decltype(more)::value) {  // (in this order: a wait for one tile leaves the later ones in flight)
                __builtin_amdgcn_sched_barrier(0);
                load_tile(next, min(item_next, items - 1), pass_next, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < GS; ++r) {
                // (a group past the wave's share meets zeros: its codes are finite, but its scale need not be)
                const bool in = r < share && (pass * kMvWaves + wave) * share + r < KG;
                const uint32_t u[4] = {b.w[r][j].x, b.w[r][j].y, b.w[r][j].z, b.w[r][j].w};
                floatx4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f16x8 q = codes(u[e]);
#pragma unroll
                    for (int k = NP - 1; k >= 0; --k) z = __builtin_amdgcn_mfma_f32_16x16x32_f16(xt[r][e][k], q, z, 0, 0, 0);
                }
                const float s = in ? dev::bf16_bits_to_float(b.sc[r][j]) : 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[q] = fmaf(s, z[q], acc[q]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[j][q] = (pass ? sum[j][q] : 0.f) + ldexpf(acc[q], back[q]);
        }
        if (last) {
            // The waves' sums are added in wave order.
            if (LOOP && item != first) lds_barrier();
#pragma unroll
            for (int j = 0; j < RB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) red[((wave * RB + j) * 4 + q) * kWave + lane] = sum[j][q];
            lds_barrier();
            if (mine) {
                float total = 0.f;
#pragma unroll
                for (int k = ONE ? 1 : 0; k >= 0; --k) {
                    const int pr = k * T + o_token;  // row of the product
                    float part = 0.f;
#pragma unroll
                    for (int v = 0; v < kMvWaves; ++v)
                        part += red[((v * RB + o_row / 16) * 4 + (pr & 3)) * kWave + (pr >> 2) * 16 + (o_row & 15)];
                    total += part;
                }
                float inv = 1.f, squared = 0.f;
                if constexpr (PRE) inv = pre.inv[o_token];
                else if (norm) {
#pragma unroll
                    for (int v = 0; v < kMvWaves; ++v) squared += sq[v][o_token];
                    inv = rsqrtf(squared / float(K) + 1e-6f);
                }
                total *= inv;
                if (!finite(total) || inv == 0.f) {  // (0 where the squares' sum is infinite)
                    const float *xr = x + size_t(o_token) * K;
                    if (!PRE && norm) inv = norm_factor(squared, xr, K);
                    total = row_dot(w + size_t(row) * (K / 2), scales + size_t(row) * KG, xr, inv, K);
                }
                y[at] = add ? addend + total : total;
            }
        }
        item = item_next;
        pass = pass_next;
    };
    if constexpr (LOOP) {
        // (pairs without a way out between them: the compiler would take the weights in flight for needed there)
        int left = (items - first + int(gridDim.x) - 1) / int(gridDim.x) * passes;
#pragma unroll 1
        for (; left >= 2; left -= 2) {
            unit(b0, b1, std::true_type());
            unit(b1, b0, std::true_type());
        }
        if (left) unit(b0, b1, std::false_type());
    } else {
        unit(b0, b1, std::false_type());
    }
}

// Many rows: every wave takes RB row tiles over all the columns, with no barrier or sum between waves; the tokens'
// terms are formed once per block and lie in LDS for all its waves.  The groups go by fours, the weights of two in
// flight while two are multiplied; the two are loaded together, since they share their lines.
constexpr int stream_lds(int T, int K) { return K * 4 * T; }

template <int RB, bool ONE>
__global__ __launch_bounds__(kMvBlock, 2) void matvec_stream_kernel(const float *__restrict__ x, const uint8_t *__restrict__ w,
                                                                    int T, int N, int K, const float *add, float *y,
                                                                    bool norm, int items) {
    constexpr int NP = ONE ? 1 : 2;  // products
    extern __shared__ uint4 lds[];
    __shared__ float inv_sh[16];
    __shared__ int exps[16];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, n = lane & 15, c = lane >> 4;
    const int KG = K / 128, waves = gridDim.x * kMvWaves;
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(w + size_t(N) * (K / 2));

    uint4 wv[4][RB];
    uint2 sc[RB];  // the scales of four groups
    const uint8_t *wrow[RB];
    const uint16_t *srow[RB];
    auto load_pair = [&](int pair, int g) __attribute__((always_inline)) {  // (past the end: loaded, not used)
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            wv[2 * pair][j] = dev::load16(wrow[j] + size_t(min(g, KG - 1)) * 64);
            wv[2 * pair + 1][j] = dev::load16(wrow[j] + size_t(min(g + 1, KG - 1)) * 64);
        }
    };
    auto load_scales = [&](int g) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            if (KG % 4 == 0) sc[j] = *reinterpret_cast<const uint2 *>(srow[j] + min(g, KG - 4));
            else {
                uint32_t v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = srow[j][min(g + r, KG - 1)];
                sc[j] = make_uint2(v[0] | (v[1] << 16), v[2] | (v[3] << 16));
            }
        }
    };
    auto start = [&](int item) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const size_t row = min((min(item, items - 1) * RB + j) * 16 + n, N - 1);
            wrow[j] = w + row * (K / 2) + 16 * c;
            srow[j] = scales + row * KG;
        }
        load_scales(0);
        load_pair(0, 0);
        load_pair(1, 2);
    };
    int item = blockIdx.x * kMvWaves + wave;
    start(item);

    // Tokens wave, wave + 8: largest magnitude and sum of squares, then the terms (256 columns per step).
#pragma unroll 1
    for (int t = wave; t < T; t += kMvWaves) {
        const float4 *xr = reinterpret_cast<const float4 *>(x + size_t(t) * K) + lane;
        float top = 0.f, squares = 0.f;
#pragma unroll 4
        for (int i = lane; i < K / 4; i += kWave) {
            const float4 u = dev::load_f4(xr + (i - lane));
            top = fmaxf(top, top_of(u));
            squares += squares_of(u);
        }
        top = wave_top(top);
        squares = dev::wave_sum(squares);
        const int e2 = exponent_of(top);
        if (lane == 0) {
            exps[t] = -kCodeExp - e2;
            inv_sh[t] = norm ? norm_factor(squares, x + size_t(t) * K, K) : 1.f;
        }
#pragma unroll 4
        for (int i = lane; i < K / 4; i += kWave) {  // (K / 4 is a multiple of 32: a pair of lanes stays together)
            uint4 *f = lds + ((i >> 5) * 16 + ((i >> 1) & 3) * 4 + ((i >> 3) & 3)) * (2 * T) + t;
            store_terms(dev::load_f4(xr + (i - lane)), e2, lane & 1, [&](int k) { return f + k * T; });
        }
    }
    __syncthreads();
    // Rows of the product: ONE: token n % 8, term n / 8; otherwise token n, one product per term.  (Rows past the last
    // token repeat it and are not stored.)
    const uint4 *xf = lds + c * (2 * T) + (ONE ? (n >> 3) * T + min(n & 7, T - 1) : min(n, T - 1));

#pragma unroll 1
    for (; item < items; item += waves) {
        floatx4 acc[RB];
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        uint2 now[RB];
        auto group = [&](int slot, int g) __attribute__((always_inline)) {
            f16x8 xt[4][NP];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int k = 0; k < NP; ++k) xt[e][k] = __builtin_bit_cast(f16x8, xf[(g * 16 + e * 4) * (2 * T) + k * T]);
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const uint32_t u[4] = {wv[slot][j].x, wv[slot][j].y, wv[slot][j].z, wv[slot][j].w};
                floatx4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f16x8 q = codes(u[e]);
#pragma unroll
                    for (int k = NP - 1; k >= 0; --k) z = __builtin_amdgcn_mfma_f32_16x16x32_f16(xt[e][k], q, z, 0, 0, 0);
                }
                const uint32_t pair = slot & 2 ? now[j].y : now[j].x;
                const float s = __uint_as_float(slot & 1 ? pair & 0xffff0000u : pair << 16);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[j][q] = fmaf(s, z[q], acc[j][q]);
            }
        };
        int g = 0;
#pragma unroll 1
        for (; g + 3 < KG; g += 4) {
#pragma unroll
            for (int j = 0; j < RB; ++j) now[j] = sc[j];
            __builtin_amdgcn_sched_barrier(0);
            load_scales(g + 4);
            group(0, g);
            group(1, g + 1);
            __builtin_amdgcn_sched_barrier(0);
            load_pair(0, g + 4);
            __builtin_amdgcn_sched_barrier(0);
            group(2, g + 2);
            group(3, g + 3);
            __builtin_amdgcn_sched_barrier(0);
            load_pair(1, g + 6);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < RB; ++j) now[j] = sc[j];
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (g + r < KG) group(r, g + r);
        if (item + waves < items) start(item + waves);
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const int row = (item * RB + j) * 16 + n;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v = acc[j][q];
                if constexpr (ONE) {  // the two terms of a token lie in rows 8 apart: lanes 32 apart
                    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
                    v = __uint_as_float(r[1]) + __uint_as_float(r[0]);
                }
                const int t = 4 * c + q;
                if (t >= T || row >= N) continue;  // (ONE: t < T <= 8 leaves lanes 0-31)
                const float inv = inv_sh[t];
                v = ldexpf(v, exps[t]) * inv;
                if (!finite(v)) v = row_dot(w + size_t(row) * (K / 2), scales + size_t(row) * KG, x + size_t(t) * K, inv, K);
                const size_t at = size_t(t) * N + row;
                y[at] = add ? add[at] + v : v;
            }
        }
    }
}

template <int RB, int GS, bool ONE, bool MULTI, bool PRE>
hipError_t run(const float *x, const uint8_t *w, int T, int N, int K, const float *add, float *y, bool norm, void *ws,
               hipStream_t s) {
    const int tiles = (N + 15) / 16, items = (tiles + RB - 1) / RB;
    // one item per block where they fit the device together, else persistent blocks (rows enough for those at K up to 2048
    // go to the other kernel)
    const int lds = lds_bytes(PRE ? 0 : T, GS, RB);
    if constexpr (MULTI || GS == 4) {
        if (MULTI || items > kMvFit) {
            matvec_int4_kernel<RB, GS, ONE, MULTI, true, PRE><<<items <= kMvFit ? items : kMvGrid, kMvBlock, lds, s>>>(x, w, T, N, K, add, y, norm, items, ws);
            return hipGetLastError();
        }
    }
    if constexpr (!MULTI) matvec_int4_kernel<RB, GS, ONE, false, false, PRE><<<items, kMvBlock, lds, s>>>(x, w, T, N, K, add, y, norm, items, ws);
    return hipGetLastError();
}

}  // namespace

size_t matvec_int4_workspace_bytes(int T, int K) { return T <= kMvTokens ? 0 : 256 + size_t(4) * T * K; }

hipError_t launch_matvec_int4(const float *x, const void *w, int T, int N, int K, const float *add, float *y, bool norm,
                              void *ws, hipStream_t s) {
    const auto *wb = static_cast<const uint8_t *>(w);
    const int tiles = (N + 15) / 16;
    // A wave per row tile takes time by K, the columns shared by a block's waves time by N.  Taken with a tile for every wave
    // that fits the device (131071 x 2048, 3 tokens: 33.7 us, 43.0 shared; 30000 x 8192, 1 token 40.5 and 40.4), and down
    // to a quarter of that where rows are many times the columns (1 token: 12000 x 512 7.0 and 7.4 us; 20000 x 2048 10.6 and
    // 9.5, the first blocks having all the tiles there; 12000 x 2048 10.3 and 7.4, 20000 x 4096 18.9 and 14.9, which are
    // shared).
    const bool many = tiles >= kMvGrid * kMvWaves || (tiles >= kMvGrid * kMvWaves / 4 && N / 8 >= K);
    if (many && stream_lds(T, K) <= 128 * 1024) {
        // two blocks per unit where the tokens' terms and a wave's registers leave room, else more tiles per wave
        const int per = T <= 8 && stream_lds(T, K) <= 72 * 1024 ? 2 : 1, waves = per * kMvGrid * kMvWaves;
        const int rb = tiles >= 4 * waves && per == 1 ? 4 : tiles >= 2 * waves ? 2 : 1, items = (tiles + rb - 1) / rb;
#define STREAM(RB, ONE) \
    if (rb == RB && (T <= 8) == ONE) matvec_stream_kernel<RB, ONE><<<per * kMvGrid, kMvBlock, stream_lds(T, K), s>>>(x, wb, T, N, K, add, y, norm, items);
        STREAM(1, true) STREAM(2, true) STREAM(4, true) STREAM(1, false) STREAM(2, false) STREAM(4, false)
#undef STREAM
        return hipGetLastError();
    }
    const bool pre = T > kMvTokens;
    if (pre) {
        matvec_terms_kernel<<<T, kTermsBlock, 0, s>>>(x, T, K, norm, static_cast<uint8_t *>(ws));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // Four groups per wave where K has more than two for each of the eight waves; with more than eight tokens, whose terms
    // fill the registers, where that makes one pass over the columns (16 tokens: 40000 x 4096 33 us, 42 in two passes of two
    // groups; 20000 x 8192 58 us in two of four, 47 in four of two).
    const int gs = K <= 2048 || (T > 8 && K > 4096) ? 2 : 4;
    const int rb = tiles <= kMvFit ? 1 : 2;
    const bool multi = K > kMvWaves * gs * 128;
#define MATVEC(RB, GS, ONE, MULTI, PRE)                                                 \
    if (rb == RB && gs == GS && (T <= 8) == ONE && multi == MULTI && pre == PRE)        \
        return run<RB, GS, ONE, MULTI, PRE>(x, wb, T, N, K, add, y, norm, ws, s);
    MATVEC(1, 2, true, false, false) MATVEC(2, 2, true, false, false)
    MATVEC(1, 4, true, false, false) MATVEC(2, 4, true, false, false) MATVEC(1, 4, true, true, false) MATVEC(2, 4, true, true, false)
    MATVEC(1, 2, true, false, true) MATVEC(2, 2, true, false, true)
    MATVEC(1, 4, true, false, true) MATVEC(2, 4, true, false, true) MATVEC(1, 4, true, true, true) MATVEC(2, 4, true, true, true)
    MATVEC(1, 2, false, false, true) MATVEC(2, 2, false, false, true) MATVEC(1, 4, false, false, true) MATVEC(2, 4, false, false, true) MATVEC(1, 2, false, true, true) MATVEC(2, 2, false, true, true)
#undef MATVEC
    return hipErrorInvalidValue;
}

}  // namespace moe
