// kv4_attention.hip -- attention over the 4-bit cache (layout in kv4.h), one or many tokens per sequence.
//
// With K = s_g u + m_g per group g of 64 dims, q . K_p = sum_g s_gp (q_g . u_gp) + m_gp (sum of q_g): the codes
// enter the matrix products as they are (bf16 of 16 + u is one shift and one bit operation for two codes; the
// products start at -16 times the sum of q_g), and the scales multiply fp32 sums of exact products.  The value
// side is sum_p (P_p s_gp) u_p + P_p m_gp.  Scores are formed transposed (positions x rows), so that a lane
// holds one row's probabilities of the positions that are its operand of the value product (P stays in
// registers), and the outputs as dims x rows, so that a row's running maximum and sum belong to its lane.
//
// A row is a (token, query head of the group) pair; a wave takes NT tiles of 16 rows over every fourth block
// of 32 positions, and the block's waves join their (max, sum, output) through LDS.  With few rows the
// positions are split over more blocks (grid), whose partial results a second launch joins.
#include "device_common.h"
#include "internal.h"
#include "kv4.h"

#include <algorithm>

namespace moe {
namespace {

using namespace kv4;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kAttWaves = 4, kAttBlock = 64 * kAttWaves;
constexpr int kMaxSplits = 128;

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ bf16x8 operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d));
}
// bf16 16 + u of a word's eight codes: 16 is 0x4180, its mantissa's lowest bit but three is worth one.
__device__ __forceinline__ bf16x8 codes16(uint32_t w) {
    constexpr uint32_t M = 0x00780078u, B = 0x41804180u;
    return operand(((w << 3) & M) | B, ((w >> 1) & M) | B, ((w >> 5) & M) | B, ((w >> 9) & M) | B);
}
constexpr uint32_t kMinus16 = 0xC180C180u;  // bf16 -16 twice

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // round to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {__bf16(lo), __bf16(hi)};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight fp32 values as TERMS bf16 operands, each rounding what the ones before it leave (one term: the
// rounded values, within 2^-8; two terms leave at most 2^-16 of a value, three nothing of its 24 bits).
template <int TERMS>
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&t)[TERMS]) {
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16(r[2 * e], r[2 * e + 1]);
            if (k + 1 < TERMS) {
                r[2 * e] -= low_half(w[e]);
                r[2 * e + 1] -= high_half(w[e]);
            }
        }
        t[k] = operand(w[0], w[1], w[2], w[3]);
    }
}

struct AttendArgs {
    const void *q;
    void *out;
    const uint8_t *cache;
    float *part;  // [T][heads][splits][d + 4]: unnormalised output, maximum, sum (more than one split)
    long long q_stride, out_stride;
    int n_heads, n_kv, group, window, splits;
    float scale;  // times log2(e)
    Batch batch;
    int *err;
};

// grid: (splits x row tiles, key/value head, sequence)
template <int NG, int NT, bool F32>
__global__ __launch_bounds__(kAttBlock) void kv4_attend_kernel(AttendArgs a) {
    constexpr int d = NG * kGroup, QT = F32 ? 3 : 1, PT = F32 ? 2 : 1;
    __shared__ float4 out_sh[kAttWaves][16][d / 4 + 1];
    __shared__ float max_sh[kAttWaves][16], sum_sh[kAttWaves][16];
    const Seq s = sequence(a.batch, blockIdx.z);
    const int h = blockIdx.y, split_i = blockIdx.x % a.splits, tile = blockIdx.x / a.splits;
    if (s.bad && blockIdx.x == 0 && h == 0 && threadIdx.x == 0) atomicOr(a.err, kErrRange);
    const int G = a.group, rows = s.n * G, row0 = tile * 16 * NT;
    if (row0 >= rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4;

    // The tile's rows: their queries as operands (k = dims), their last visible position.
    int last[NT];
    bf16x8 bq[NT][2 * NG][QT], bm[NT];
    floatx4 init[NT][NG];  // -16 sum of q_g
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = row0 + 16 * t + n, i = row / G, head = h * G + row % G;
        const bool live = row < rows;
        last[t] = live ? s.len - s.n + i : -1;
        const size_t at = live ? size_t(s.t0 + i) * a.q_stride + size_t(head) * d : 0;
#pragma unroll
        for (int j = 0; j < 2 * NG; ++j) {
            if constexpr (F32) {
                float x[8];
                const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(a.q) + at + 32 * j + 8 * c);
                float4 u = make_float4(0.f, 0.f, 0.f, 0.f), v = u;
                if (live) u = dev::load_f4(p), v = dev::load_f4(p + 1);
                x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
                split<QT>(x, bq[t][j]);
            } else {
                uint4 u = make_uint4(0, 0, 0, 0);
                if (live) u = dev::load16(reinterpret_cast<const uint8_t *>(static_cast<const uint16_t *>(a.q) + at + 32 * j + 8 * c));
                bq[t][j][0] = __builtin_bit_cast(bf16x8, u);
            }
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            floatx4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = QT - 1; k >= 0; --k)
#pragma unroll
                for (int j = 2 * g; j < 2 * g + 2; ++j)
                    z = mfma(operand(kMinus16, kMinus16, kMinus16, kMinus16), bq[t][j][k], z);
            init[t][g] = z;
        }
        // The bases' product: elements (c, 0..2) are the three terms of the sum of q over group c.
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) sum = c == g ? init[t][g][0] * -0.0625f : sum;
        const float x[8] = {sum, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        bf16x8 w[3];
        split<3>(x, w);
        const uint32_t w0 = __builtin_bit_cast(uint4, w[0]).x, w1 = __builtin_bit_cast(uint4, w[1]).x;
        bm[t] = operand((w0 & 0xffffu) | (w1 << 16), __builtin_bit_cast(uint4, w[2]).x & 0xffffu, 0, 0);
    }

    // Blocks of positions: those that some row of the tile sees, this split's share of them.
    const int p_first = s.len - s.n + row0 / G;                               // of the tile's first row
    const int p_last = s.len - s.n + min(s.n - 1, (row0 + 16 * NT - 1) / G);  // of its last row
    const int b_first = a.window ? max(0, p_first - a.window + 1) / kPos : 0;
    const int b_end = p_last < 0 ? b_first : p_last / kPos + 1;
    const int share = max((b_end - b_first + a.splits - 1) / a.splits, kAttWaves);
    const int b0 = b_first + split_i * share, b1 = min(b_end, b0 + share);
    const uint8_t *seq = a.cache + (size_t(blockIdx.z) * a.n_kv + h) * (a.batch.max_pos / kPos) * block_bytes(d);

    floatx4 acc[NT][4 * NG], add[NT][NG];  // outputs (dims x rows); what all the dims of a group share
    float mx[NT], sum[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        mx[t] = -INFINITY;
        sum[t] = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * NG; ++i) acc[t][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < NG; ++g) add[t][g] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll 1
    for (int b = b0 + wave; b < b1; b += kAttWaves) {
        const uint8_t *block = seq + size_t(b) * block_bytes(d);
        uint4 kc[NG], vc[NG], ks[NG], vs[NG], vm[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            kc[g] = dev::load16(block + k_codes(d) + g * 1024 + lane * 16);
            ks[g] = dev::load16(block + k_scales(d) + g * 64 + c * 16);
            vc[g] = dev::load16(block + v_codes(d) + g * 1024 + lane * 16);
            vs[g] = dev::load16(block + v_scales(d) + g * 64 + c * 16);
            vm[g] = dev::load16(block + v_bases(d) + g * 64 + c * 16);
        }
        const uint32_t km = *reinterpret_cast<const uint32_t *>(block + k_bases(d) + min(c, NG - 1) * 64 + n * 4);
        if (b * kPos + kPos > s.len) {
            // Positions that hold nothing yet may hold anything: their probabilities are 0, and 0 times what
            // lies there has to be 0.
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t keep = 0;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int k = 2 * i + e, p = b * kPos + 16 * (k >> 2) + 4 * c + (k & 3);
                    keep |= p < s.len ? 0xffffu << (16 * e) : 0u;
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    reinterpret_cast<uint32_t *>(&vs[g])[i] &= keep;
                    reinterpret_cast<uint32_t *>(&vm[g])[i] &= keep;
                }
            }
        }
        bf16x8 kf[2][2 * NG], vf[4 * NG];
#pragma unroll
        for (int w = 0; w < 4 * NG; ++w) {
            kf[w / (2 * NG)][w % (2 * NG)] = codes16(reinterpret_cast<const uint32_t *>(&kc[w / 4])[w % 4]);
            vf[w] = codes16(reinterpret_cast<const uint32_t *>(&vc[w / 4])[w % 4]);
        }
        const bool full = b * kPos + kPos - 1 <= p_first && (!a.window || b * kPos > p_last - a.window);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float x[8];
#pragma unroll
            for (int tau = 0; tau < 2; ++tau) {
                const uint32_t m2 = tau ? (km >> 16) * 0x10001u : (km & 0xffffu) * 0x10001u;
                floatx4 z = mfma(operand(m2, m2, m2, m2), bm[t], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    floatx4 y = init[t][g];
#pragma unroll
                    for (int k = QT - 1; k >= 0; --k)
#pragma unroll
                        for (int j = 2 * g; j < 2 * g + 2; ++j) y = mfma(kf[tau][j], bq[t][j][k], y);
                    const uint32_t *sc = reinterpret_cast<const uint32_t *>(&ks[g]) + 2 * tau;
                    z[0] = fmaf(low_half(sc[0]), y[0], z[0]);
                    z[1] = fmaf(high_half(sc[0]), y[1], z[1]);
                    z[2] = fmaf(low_half(sc[1]), y[2], z[2]);
                    z[3] = fmaf(high_half(sc[1]), y[3], z[3]);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) x[4 * tau + r] = z[r] * a.scale;
            }
            if (!full) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int p = b * kPos + 16 * (k >> 2) + 4 * c + (k & 3);
                    if (p > last[t] || (a.window && p <= last[t] - a.window)) x[k] = -INFINITY;
                }
            }
            float top = x[0];
#pragma unroll
            for (int k = 1; k < 8; ++k) top = fmaxf(top, x[k]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float was = mx[t], now = fmaxf(was, top);
            if (__any(now > was)) {  // some row's maximum rose: what it has so far is scaled down
                const float f = was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(was - now);
                mx[t] = now;
                sum[t] *= f;
#pragma unroll
                for (int i = 0; i < 4 * NG; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][i][r] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int r = 0; r < 4; ++r) add[t][g][r] *= f;
            }
            const float base = now == -INFINITY ? 0.f : now;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[k] = __builtin_amdgcn_exp2f(x[k] - base);
                sum[t] += x[k];
            }
            bf16x8 bp[PT];
            split<PT>(x, bp);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float y[8];
                const uint32_t *sc = reinterpret_cast<const uint32_t *>(&vs[g]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[2 * e] = x[2 * e] * low_half(sc[e]);
                    y[2 * e + 1] = x[2 * e + 1] * high_half(sc[e]);
                }
                bf16x8 bs[PT];
                split<PT>(y, bs);
#pragma unroll
                for (int k = PT - 1; k >= 0; --k) {
                    add[t][g] = mfma(__builtin_bit_cast(bf16x8, vm[g]), bp[k], add[t][g]);
                    add[t][g] = mfma(operand(kMinus16, kMinus16, kMinus16, kMinus16), bs[k], add[t][g]);
#pragma unroll
                    for (int i = 4 * g; i < 4 * g + 4; ++i) acc[t][i] = mfma(vf[i], bs[k], acc[t][i]);
                }
            }
        }
    }

    // Join the waves, one tile of rows at a time.
#pragma unroll 1
    for (int t = 0; t < NT; ++t) {
        floatx4 o[4 * NG];
        float m = 0.f, l = 0.f;
#pragma unroll
        for (int u = 0; u < NT; ++u)
            if (u == t) {
                m = mx[u];
                l = sum[u];
#pragma unroll
                for (int i = 0; i < 4 * NG; ++i) o[i] = acc[u][i] + add[u][i / 4];
            }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (t) __syncthreads();
        if (c == 0) {
            max_sh[wave][n] = m;
            sum_sh[wave][n] = l;
        }
#pragma unroll
        for (int i = 0; i < 4 * NG; ++i) out_sh[wave][n][4 * i + c] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
        __syncthreads();
#pragma unroll 1
        for (int idx = threadIdx.x; idx < 16 * (d / 4); idx += kAttBlock) {
            const int r = idx / (d / 4), i4 = idx % (d / 4), row = row0 + 16 * t + r;
            if (row >= rows) continue;
            float M = max_sh[0][r];
#pragma unroll
            for (int w = 1; w < kAttWaves; ++w) M = fmaxf(M, max_sh[w][r]);
            float S = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kAttWaves; ++w) {
                // (a wave that saw nothing of the row has the maximum -inf and the sum 0; one whose scores are
                // all NaN has the sum NaN, which stays)
                const float f = max_sh[w][r] == -INFINITY && sum_sh[w][r] == 0.f ? 0.f : __builtin_amdgcn_exp2f(max_sh[w][r] - M);
                const float4 u = out_sh[w][r][i4];
                S = fmaf(f, sum_sh[w][r], S);
                v.x = fmaf(f, u.x, v.x);
                v.y = fmaf(f, u.y, v.y);
                v.z = fmaf(f, u.z, v.z);
                v.w = fmaf(f, u.w, v.w);
            }
            const int i = row / G, head = h * G + row % G;
            const size_t token = size_t(s.t0 + i);
            if (a.splits > 1) {
                float *p = a.part + ((token * a.n_heads + head) * a.splits + split_i) * (d + 4);
                *reinterpret_cast<float4 *>(p + 4 * i4) = v;
                if (i4 == 0) *reinterpret_cast<float2 *>(p + d) = make_float2(M, S);
                continue;
            }
            const float inv = S == 0.f ? 0.f : 1.f / S;  // (a row that sees nothing: 0)
            v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
            const size_t at = token * a.out_stride + size_t(head) * d + 4 * i4;
            if constexpr (F32) *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = v;
            else
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) =
                    make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        }
    }
}

// Joins the splits of one row.  grid: (rows, key/value head, sequence); 8 groups of d / 4 lanes (at most 64)
// take the splits in turn.
template <int NG, bool F32>
__global__ __launch_bounds__(kAttBlock) void kv4_join_kernel(AttendArgs a) {
    constexpr int d = NG * kGroup, N4 = d / 4, SUB = kAttBlock / N4;
    __shared__ float wgt[kMaxSplits], red[2 * kAttWaves];
    __shared__ float4 acc_sh[SUB][N4];
    const Seq s = sequence(a.batch, blockIdx.z);
    const int G = a.group, row = blockIdx.x, h = blockIdx.y;
    if (row >= s.n * G) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const size_t token = size_t(s.t0 + row / G);
    const int head = h * G + row % G;
    const float *p = a.part + (token * a.n_heads + head) * a.splits * (d + 4);
    float m = -INFINITY, l = 0.f;
    if (tid < a.splits) {
        const float2 ml = *reinterpret_cast<const float2 *>(p + size_t(tid) * (d + 4) + d);
        m = ml.x;
        l = ml.y;
    }
    float M = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    if (lane == 0) red[wave] = M;
    __syncthreads();
    M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float f = m == -INFINITY && l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - M);
    if (tid < a.splits) wgt[tid] = f;
    const float S1 = dev::wave_sum(f * l);
    if (lane == 0) red[kAttWaves + wave] = S1;
    __syncthreads();
    const float S = red[kAttWaves] + red[kAttWaves + 1] + red[kAttWaves + 2] + red[kAttWaves + 3];
    const int i4 = tid % N4, sub = tid / N4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (sub < SUB) {
        for (int k = sub; k < a.splits; k += SUB) {
            const float w = wgt[k];
            if (w == 0.f) continue;
            const float4 u = *reinterpret_cast<const float4 *>(p + size_t(k) * (d + 4) + 4 * i4);
            v.x = fmaf(w, u.x, v.x);
            v.y = fmaf(w, u.y, v.y);
            v.z = fmaf(w, u.z, v.z);
            v.w = fmaf(w, u.w, v.w);
        }
        acc_sh[sub][i4] = v;
    }
    __syncthreads();
    if (tid >= N4) return;
    v = acc_sh[0][tid];
#pragma unroll
    for (int k = 1; k < SUB; ++k) {
        const float4 u = acc_sh[k][tid];
        v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
    }
    const float inv = S == 0.f ? 0.f : 1.f / S;
    v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
    const size_t at = token * a.out_stride + size_t(head) * d + 4 * tid;
    if constexpr (F32) *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = v;
    else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// Tiles of 16 rows per wave, and the splits of the positions.
struct AttendPlan {
    int tiles, blocks, splits;
};
AttendPlan attend_plan(int n_seq, int n_kv, int group, int d, int max_q, int max_pos, bool f32) {
    const long long rows = (long long)max_q * group;
    const int most = d <= 128 ? (f32 ? 2 : 4) : (f32 ? 1 : 2);  // what a wave's registers hold
    AttendPlan p;
    p.tiles = rows <= 16 ? 1 : rows <= 32 ? std::min(2, most) : most;
    p.blocks = int((rows + 16 * p.tiles - 1) / (16 * p.tiles));
    const long long base = (long long)p.blocks * n_kv * n_seq;
    const long long most_splits = std::max(1, max_pos / kPos / kAttWaves);
    p.splits = int(std::max(1ll, std::min({(long long)kMaxSplits, most_splits, 512 / base})));
    return p;
}

}  // namespace

size_t kv4_attention_workspace_bytes(int T, int n_seq, int n_heads, int n_kv, int d, int max_q, int max_pos) {
    size_t n = 0;
    for (bool f32 : {false, true}) {
        const AttendPlan p = attend_plan(n_seq, n_kv, n_heads / n_kv, d, max_q, max_pos, f32);
        if (p.splits > 1) n = std::max(n, size_t(T) * n_heads * p.splits * (d + 4) * sizeof(float));
    }
    return (n + 255) & ~size_t(255);
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
    a.splits = p.splits;
    a.scale = scale * 1.44269504088896341f;
    a.batch = batch;
    a.err = err;
    const dim3 grid(p.blocks * p.splits, n_kv, batch.n_seq);
#define KV4_RUN(NG, NT, F) kv4_attend_kernel<NG, NT, F><<<grid, kAttBlock, 0, s>>>(a)
#define KV4_SMALL(NG)                               \
    case NG * kGroup:                               \
        if (f32) {                                  \
            if (p.tiles == 1) KV4_RUN(NG, 1, true); \
            else KV4_RUN(NG, 2, true);              \
        } else {                                    \
            if (p.tiles == 1) KV4_RUN(NG, 1, false); \
            else if (p.tiles == 2) KV4_RUN(NG, 2, false); \
            else KV4_RUN(NG, 4, false);             \
        }                                           \
        break;
#define KV4_LARGE(NG)                               \
    case NG * kGroup:                               \
        if (f32) KV4_RUN(NG, 1, true);              \
        else if (p.tiles == 1) KV4_RUN(NG, 1, false); \
        else KV4_RUN(NG, 2, false);                 \
        break;
    switch (d) {
        KV4_SMALL(1) KV4_SMALL(2) KV4_LARGE(3) KV4_LARGE(4)
    default: return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const dim3 jgrid(batch.max_q * a.group, n_kv, batch.n_seq);
#define KV4_JOIN(NG)                                                    \
    case NG * kGroup:                                                   \
        if (f32) kv4_join_kernel<NG, true><<<jgrid, kAttBlock, 0, s>>>(a); \
        else kv4_join_kernel<NG, false><<<jgrid, kAttBlock, 0, s>>>(a); \
        break;
    switch (d) { KV4_JOIN(1) KV4_JOIN(2) KV4_JOIN(3) KV4_JOIN(4) }
#undef KV4_JOIN
#undef KV4_LARGE
#undef KV4_SMALL
#undef KV4_RUN
    return hipGetLastError();
}

}  // namespace moe
