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
// A block takes items of RB row tiles; its eight waves share the columns and keep their part of the tokens in
// registers from item to item, with the next item's weights in flight.
#include "device_common.h"
#include "internal.h"

namespace moe {
namespace {

using dev::kWave;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kMvWaves = 8, kMvBlock = kMvWaves * kWave;
constexpr int kMvGrid = 256;  // persistent blocks: one per compute unit
constexpr int kCodeExp = -9;

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

// GS: quantisation groups per wave and pass.  ONE: the two terms share one product (rows term * T + token).
template <int RB, int GS, bool ONE, bool NORM>
__global__ __launch_bounds__(kMvBlock, 2) void matvec_int4_kernel(const float *__restrict__ x, const uint8_t *__restrict__ w,
                                                                  int T, int N, int K, const float *add, float *y,
                                                                  int items) {
    constexpr int NP = ONE ? 1 : 2;  // products
    __shared__ float red[2][kMvWaves][RB][4][kWave];
    __shared__ float sq[kMvWaves][16], inv_sh[16];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, n = lane & 15, c = lane >> 4;
    const int KG = K / 128, passes = (KG + kMvWaves * GS - 1) / (kMvWaves * GS);
    const int share = (KG + kMvWaves * passes - 1) / (kMvWaves * passes);  // groups per wave and pass, <= GS
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(w + size_t(N) * (K / 2));
    // (rows past the last token repeat it and are not stored)
    const int token = min(ONE && n >= T ? n - T : n, T - 1);
    const bool second = ONE && n >= T;

    struct Weights {
        uint4 w[GS][RB];
        uint32_t sc[GS][RB];
    } b0, b1;
    auto group = [&](int pass, int r) { return (pass * kMvWaves + wave) * share + r; };
    auto load_w = [&](Weights &b, int item, int pass) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < GS; ++r) {
            const int g = min(group(pass, min(r, share - 1)), KG - 1);  // (past the end: loaded, not used)
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const size_t row = min((item * RB + j) * 16 + n, N - 1);
                b.w[r][j] = dev::load16_stream(w + row * (K / 2) + size_t(g) * 64 + 16 * c);
                b.sc[r][j] = scales[row * KG + g];
            }
        }
    };
    float4 raw[GS][8];
    auto load_x = [&](int pass) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < GS; ++r) {
            const int g = min(group(pass, min(r, share - 1)), KG - 1);
            const float4 *p = reinterpret_cast<const float4 *>(x + size_t(token) * K + g * 128 + 32 * c);
#pragma unroll
            for (int j = 0; j < 8; ++j) raw[r][j] = dev::load_f4(p + j);
        }
    };
    float top = 0.f, squares = 0.f;
    auto measure = [&](int pass) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < GS; ++r) {
            if (r >= share || group(pass, r) >= KG) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 v = raw[r][j];
                top = fmaxf(fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
                if (NORM) squares = fmaf(v.x, v.x, fmaf(v.y, v.y, fmaf(v.z, v.z, fmaf(v.w, v.w, squares))));
            }
        }
    };
    f16x8 xt[GS][4][NP];
    int e2 = 0;  // 2^e2 scales the token's values
    auto convert = [&](int pass) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < GS; ++r) {
            const bool in = r < share && group(pass, r) < KG;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 a = raw[r][2 * j], b = raw[r][2 * j + 1];
                const float v[8] = {a.x, b.x, a.y, b.y, a.z, b.z, a.w, b.w};  // the codes' order
                f16x2 hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float u0 = in ? ldexpf(v[2 * e], e2) : 0.f, u1 = in ? ldexpf(v[2 * e + 1], e2) : 0.f;
                    hi[e] = f16x2{_Float16(u0), _Float16(u1)};
                    lo[e] = f16x2{_Float16(u0 - float(hi[e][0])), _Float16(u1 - float(hi[e][1]))};
                }
                const f16x8 h{hi[0][0], hi[0][1], hi[1][0], hi[1][1], hi[2][0], hi[2][1], hi[3][0], hi[3][1]};
                const f16x8 l{lo[0][0], lo[0][1], lo[1][0], lo[1][1], lo[2][0], lo[2][1], lo[3][0], lo[3][1]};
                if constexpr (ONE) xt[r][j][0] = second ? l : h;
                else xt[r][j][0] = h, xt[r][j][1] = l;
            }
        }
    };

    int item = blockIdx.x, pass = 0;
    load_x(0);
    load_w(b0, item, 0);
    measure(0);
#pragma unroll 1
    for (int p = 1; p < passes; ++p) {
        load_x(p);
        measure(p);
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (top > 0.f && top < INFINITY) e2 = 14 - ilogbf(top);
    if (NORM) {
        squares += __shfl_xor(squares, 16);
        squares += __shfl_xor(squares, 32);
        if (lane < 16) sq[wave][lane] = squares;
        __syncthreads();
        if (tid < T) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < kMvWaves; ++v) s += sq[v][tid];
            inv_sh[tid] = rsqrtf(s / float(K) + 1e-6f);
        }  // (read after the next barrier)
    }
    int back[4];  // what takes the sums of row 4 c + q of the product back
#pragma unroll
    for (int q = 0; q < 4; ++q) back[q] = -kCodeExp - __shfl(e2, 4 * c + q);
    if (passes == 1) convert(0);

    floatx4 acc[RB];
    int buf = 0;
    auto work = [&](Weights &b, Weights &next) __attribute__((always_inline)) {
        const bool last = pass == passes - 1;
        const int item_next = last ? item + gridDim.x : item, pass_next = last ? 0 : pass + 1;
        if (passes > 1) {
            load_x(pass);
            convert(pass);
        }
        if (item_next < items) load_w(next, item_next, pass_next);
        if (pass == 0)
#pragma unroll
            for (int j = 0; j < RB; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < GS; ++r) {
            // (a group past the wave's share meets zeros: its codes are finite, but its scale need not be)
            const bool in = r < share && group(pass, r) < KG;
#pragma unroll
            for (int j = 0; j < RB; ++j) {
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
                for (int q = 0; q < 4; ++q) acc[j][q] = fmaf(s, z[q], acc[j][q]);
            }
        }
        if (last) {
            // The waves' sums are added in wave order.  (Two buffers: one barrier per item.)
#pragma unroll
            for (int j = 0; j < RB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) red[buf][wave][j][q][lane] = ldexpf(acc[j][q], back[q]);
            __syncthreads();
            for (int o = tid; o < 16 * RB * T; o += kMvBlock) {
                const int r = o % (16 * RB), t = o / (16 * RB), row = item * 16 * RB + r;
                if (row >= N) continue;
                float sum = 0.f;
#pragma unroll
                for (int k = ONE ? 1 : 0; k >= 0; --k) {
                    const int pr = k * T + t;  // row of the product
                    float part = 0.f;
#pragma unroll
                    for (int v = 0; v < kMvWaves; ++v) part += red[buf][v][r / 16][pr & 3][(pr >> 2) * 16 + (r & 15)];
                    sum += part;
                }
                const float inv = NORM ? inv_sh[t] : 1.f;
                sum *= inv;
                if ((__float_as_uint(sum) & 0x7f800000u) == 0x7f800000u)
                    sum = row_dot(w + size_t(row) * (K / 2), scales + size_t(row) * KG, x + size_t(t) * K, inv, K);
                const size_t at = size_t(t) * N + row;
                y[at] = add ? add[at] + sum : sum;
            }
            buf ^= 1;
        }
        item = item_next;
        pass = pass_next;
    };
#pragma unroll 1
    while (true) {
        work(b0, b1);
        if (item >= items) break;
        work(b1, b0);
        if (item >= items) break;
    }
}

}  // namespace

hipError_t launch_matvec_int4(const float *x, const void *w, int T, int N, int K, const float *add, float *y, bool norm,
                              hipStream_t s) {
    const auto *wb = static_cast<const uint8_t *>(w);
    // Four groups per wave where K has more than two for each of the eight waves and the tokens' terms leave the
    // registers for it.
    const int tiles = (N + 15) / 16, gs = K <= 2048 || T > 8 ? 2 : 4;
    const bool many = tiles >= 4 * kMvGrid;
    const int rb = many ? (gs == 2 ? 4 : 2) : 1, items = (tiles + rb - 1) / rb;
    const int grid = many ? kMvGrid : items < 2 * kMvGrid ? items : 2 * kMvGrid;
#define MATVEC(RB, GS, ONE)                                                                               \
    do {                                                                                                  \
        if (norm) matvec_int4_kernel<RB, GS, ONE, true><<<grid, kMvBlock, 0, s>>>(x, wb, T, N, K, add, y, items); \
        else matvec_int4_kernel<RB, GS, ONE, false><<<grid, kMvBlock, 0, s>>>(x, wb, T, N, K, add, y, items); \
    } while (0)
    if (T <= 8) {
        if (gs == 2 && many) MATVEC(4, 2, true);
        else if (gs == 2) MATVEC(1, 2, true);
        else if (many) MATVEC(2, 4, true);
        else MATVEC(1, 4, true);
    } else {
        if (many) MATVEC(4, 2, false);
        else MATVEC(1, 2, false);
    }
#undef MATVEC
    return hipGetLastError();
}

}  // namespace moe
