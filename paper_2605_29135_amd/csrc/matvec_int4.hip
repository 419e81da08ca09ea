// matvec_int4.hip -- matrix-vector products with int4-g128 weights for 1 to 16 tokens.
//
// y[t] = add[t] + W h[t].  The bound is the weights' bytes.  On the matrix cores a 16-row tile of W is an operand
// as it lies in memory (lane l: row l % 16, 16 bytes = 32 columns of the quantisation group, quarter l / 16), so
// the work per weight does not depend on the number of tokens.  The tokens' values enter as three bf16 terms
// whose sum is exact, the codes as bf16 24 + q (one shift and one bit operation for two), with sums that start
// at -24 times the sum of x: every product is exact, and the group's scale multiplies its fp32 sum.  Up to 5
// tokens the three terms are rows of one product; for more they are three products.
#include "device_common.h"
#include "internal.h"

namespace moe {
namespace {

using dev::kWave;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kMvWaves = 8, kMvBlock = kMvWaves * kWave;
constexpr int kMvPass = 2;  // quantisation groups per wave and pass

__device__ __forceinline__ bf16x8 codes24(uint32_t w) {
    constexpr uint32_t M = 0x00780078u, B = 0x41804180u;  // 16 + unsigned nibble, 16 + (q + 8)
    const uint32_t v = w ^ 0x88888888u;
    return __builtin_bit_cast(bf16x8, make_uint4(((v << 3) & M) | B, ((v >> 1) & M) | B, ((v >> 5) & M) | B, ((v >> 9) & M) | B));
}

__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ float below(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// Term `term` of eight values in the codes' order 0,4,1,5,2,6,3,7 (a term is the top 8 bits of what the terms
// before it leave: no finite value overflows, and three terms hold all 24 bits).
__device__ __forceinline__ void split3(const float *v, bf16x8 (&t)[3]) {
    uint32_t w[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = v[e], b = v[e + 4];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            w[k][e] = high_halves(a, b);
            a = below(a);
            b = below(b);
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) t[k] = __builtin_bit_cast(bf16x8, make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]));
}

// One output in fp32, element by element: what a sum that is not finite is taken from (an infinite or huge
// value has no three terms, or its products overflow where the definition's do not).
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

// grid: persistent blocks over the items of RB tiles of 16 rows.  ONE: the three terms share one product.
template <int RB, bool ONE, bool NORM>
__global__ __launch_bounds__(kMvBlock) void matvec_int4_kernel(const float *__restrict__ x, const uint8_t *__restrict__ w,
                                                               int T, int N, int K, const float *add, float *y, int items) {
    constexpr int NP = ONE ? 1 : 3;  // products
    __shared__ float red[kMvWaves][RB][4][kWave];
    __shared__ float sq[kMvWaves][16], inv_sh[16];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, n = lane & 15, c = lane >> 4;
    const int KG = K / 128, passes = (KG + kMvWaves * kMvPass - 1) / (kMvWaves * kMvPass);
    const int share = (KG + kMvWaves * passes - 1) / (kMvWaves * passes);  // groups per wave and pass, <= kMvPass
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(w + size_t(N) * (K / 2));
    const int token = ONE ? n % T : n, term = ONE ? n / T : 0;  // of this lane's row of the product
    const bool live = ONE ? term < 3 : n < T;

    bf16x8 xt[kMvPass][4][NP];
    floatx4 init[kMvPass][ONE ? 1 : 2];  // -24 sum of x over the group: of the leading terms, of the others
    auto load_x = [&](int pass, float &squares) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < kMvPass; ++r) {
            const int g = (pass * kMvWaves + wave) * share + r;
            const bool in = live && r < share && g < KG;
            for (floatx4 &z : init[r]) z = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
                if (in) {
                    const float4 *p = reinterpret_cast<const float4 *>(x + size_t(token) * K + g * 128 + 32 * c + 8 * j);
                    a = dev::load_f4(p);
                    b = dev::load_f4(p + 1);
                }
                const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                if (NORM)
#pragma unroll
                    for (int e = 0; e < 8; ++e) squares = fmaf(v[e], v[e], squares);
                bf16x8 t[3];
                split3(v, t);
                if constexpr (ONE) xt[r][j][0] = term == 0 ? t[0] : term == 1 ? t[1] : t[2];
                else
#pragma unroll
                    for (int k = 0; k < 3; ++k) xt[r][j][k] = t[k];
                constexpr uint32_t m24 = 0xC1C0C1C0u;  // bf16 -24 twice
#pragma unroll
                for (int k = NP - 1; k >= 0; --k)
                    init[r][k > 0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        xt[r][j][k], __builtin_bit_cast(bf16x8, make_uint4(m24, m24, m24, m24)), init[r][k > 0], 0, 0, 0);
            }
        }
    };

    bool first = true;
#pragma unroll 1
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int row0 = item * 16 * RB;
        floatx4 acc[RB];
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        float squares = 0.f;
#pragma unroll 1
        for (int pass = 0; pass < passes; ++pass) {
            uint4 wv[kMvPass][RB];
            uint32_t sc[kMvPass][RB];
#pragma unroll
            for (int r = 0; r < kMvPass; ++r) {
                const int g = min((pass * kMvWaves + wave) * share + min(r, share - 1), KG - 1);
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    const size_t row = min(row0 + 16 * j + n, N - 1);
                    wv[r][j] = dev::load16_stream(w + row * (K / 2) + size_t(g) * 64 + 16 * c);
                    sc[r][j] = scales[row * KG + g];
                }
            }
            if (first || passes > 1) load_x(pass, squares);
#pragma unroll
            for (int r = 0; r < kMvPass; ++r) {
                // (a group past the wave's share meets zeros: its codes are finite, but its scale need not be)
                const bool in = r < share && (pass * kMvWaves + wave) * share + r < KG;
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    const uint32_t u[4] = {wv[r][j].x, wv[r][j].y, wv[r][j].z, wv[r][j].w};
                    // (the leading terms apart from the small ones, whose sums would be rounded at its size)
                    floatx4 z = init[r][0];
#pragma unroll
                    for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xt[r][e][0], codes24(u[e]), z, 0, 0, 0);
                    if constexpr (!ONE) {
                        floatx4 v = init[r][1];
#pragma unroll
                        for (int k = 2; k >= 1; --k)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xt[r][e][k], codes24(u[e]), v, 0, 0, 0);
                        z += v;
                    }
                    const float s = in ? dev::bf16_bits_to_float(sc[r][j]) : 0.f;
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[j][q] = fmaf(s, z[q], acc[j][q]);
                }
            }
        }
        if (NORM && first) {
            squares += __shfl_xor(squares, 16);
            squares += __shfl_xor(squares, 32);
            if (lane < 16) sq[wave][lane] = squares;
        }
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) red[wave][j][q][lane] = acc[j][q];
        __syncthreads();
        if (NORM && first) {
            if (tid < T) {
                float s = 0.f;
#pragma unroll
                for (int v = 0; v < kMvWaves; ++v) s += sq[v][tid];
                inv_sh[tid] = rsqrtf(s / float(K) + 1e-6f);
            }
            __syncthreads();
        }
        first = false;
        for (int o = tid; o < 16 * RB * T; o += kMvBlock) {
            const int r = o % (16 * RB), t = o / (16 * RB), row = row0 + r;
            if (row >= N) continue;
            float sum = 0.f;
#pragma unroll
            for (int k = ONE ? 2 : 0; k >= 0; --k) {
                const int pr = ONE ? k * T + t : t;  // row of the product
                float part = 0.f;
#pragma unroll
                for (int v = 0; v < kMvWaves; ++v) part += red[v][r / 16][pr & 3][(pr >> 2) * 16 + (r & 15)];
                sum += part;
            }
            const float inv = NORM ? inv_sh[t] : 1.f;
            sum *= inv;
            if ((__float_as_uint(sum) & 0x7f800000u) == 0x7f800000u)
                sum = row_dot(w + size_t(row) * (K / 2), scales + size_t(row) * KG, x + size_t(t) * K, inv, K);
            const size_t at = size_t(t) * N + row;
            y[at] = add ? add[at] + sum : sum;
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_matvec_int4(const float *x, const void *w, int T, int N, int K, const float *add, float *y, bool norm,
                              hipStream_t s) {
    const auto *wb = static_cast<const uint8_t *>(w);
    const int tiles = (N + 15) / 16, rb = tiles >= 4 * 512 ? 4 : 1;
    const int items = (tiles + rb - 1) / rb, grid = items < 512 ? items : 512;
#define MATVEC(RB, ONE)                                                                                   \
    do {                                                                                                  \
        if (norm) matvec_int4_kernel<RB, ONE, true><<<grid, kMvBlock, 0, s>>>(x, wb, T, N, K, add, y, items); \
        else matvec_int4_kernel<RB, ONE, false><<<grid, kMvBlock, 0, s>>>(x, wb, T, N, K, add, y, items); \
    } while (0)
    if (T <= 5) {
        if (rb == 4) MATVEC(4, true);
        else MATVEC(1, true);
    } else {
        if (rb == 4) MATVEC(4, false);
        else MATVEC(1, false);
    }
#undef MATVEC
    return hipGetLastError();
}

}  // namespace moe
