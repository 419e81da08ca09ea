// attention_int4.hip -- the decoder self-attention block of one token per sequence with int4 projections and a
// 4-bit key/value cache: the arithmetic of attention.hip's block around the quantised parts.
//
//   1. q/k/v projection with the pre-norm (matvec_int4.hip).
//   2. heads_kernel: every query and key head normalised and rotated; the new keys and values quantised into
//      the cache.
//   3. Attention over the cache (kv4_attention.hip).
//   4. Output projection added to x (matvec_int4.hip).
//
// Measured in the decode stack (H 2048, 32 query and 4 key/value heads of 128, one token; in brackets the bf16 block,
// four launches, with 3.6 times the cache and 3.9 times the weights): 21.0 us at 101 positions of a cache of 4096 (19.0;
// in a cache of 128, without the second attention launch, 18.5), 23.1 at 4096 (19.6), 24.7 at 8192 (25.9), 29.1 at 16384
// (38.2).  Up to some thousand positions five launches' latency is the bound: projections 5.5 each, heads 4.1 (fp64 rotary
// angles as in that block), attention 7 and 4.
#include "device_common.h"
#include "internal.h"
#include "kv4.h"
#include "rotary.h"

#include <math.h>

#include <algorithm>

namespace moe {
namespace {

using namespace kv4;

// One wave per (head, token): query heads in place, key/value heads into the cache.  Latency-bound: a few
// hundred bytes per wave, 4.1 us.  grid: (query heads + key/value heads, tokens)
template <int NG>
__global__ __launch_bounds__(64) void heads_kernel(float *__restrict__ qkv, int n_heads, int n_kv, float theta,
                                                   const int32_t *__restrict__ kv_len, int max_pos,
                                                   uint8_t *__restrict__ cache, int *err) {
    constexpr int d = NG * kGroup, half = d / 2, U = (half + 63) / 64;
    __shared__ float row_sh[d];
    __shared__ uint32_t code_sh[d / 8];
    const int j = blockIdx.x, t = blockIdx.y, lane = threadIdx.x;
    const int len = kv_len[t], p = len - 1;
    float *row = qkv + (size_t(t) * (n_heads + 2 * n_kv) + j) * d;
    float a[U], b[U], squares = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = lane + 64 * u;
        a[u] = i < half ? row[i] : 0.f;
        b[u] = i < half ? row[i + half] : 0.f;
        squares += a[u] * a[u] + b[u] * b[u];
    }
    const bool key = j >= n_heads;
    const float *v_row = row + size_t(n_kv) * d;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (key && lane < d / 8) {
        const float4 *q = reinterpret_cast<const float4 *>(v_row + 8 * lane);
        const float4 u = dev::load_f4(q), w = dev::load_f4(q + 1);
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = w.x, x[5] = w.y, x[6] = w.z, x[7] = w.w;
    }
    const float inv = rsqrtf(dev::wave_sum(squares) / float(d) + 1e-6f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = lane + 64 * u;
        if (i >= half) continue;
        float rc, rs;
        dev::rope_cs(p, i, d, theta, rc, rs);
        const float na = a[u] * inv, nb = b[u] * inv;
        const float ra = na * rc - nb * rs, rb = nb * rc + na * rs;
        if (key) {
            row_sh[i] = ra;
            row_sh[i + half] = rb;
        } else {
            row[i] = ra;
            row[i + half] = rb;
        }
    }
    if (!key) return;
    if (len <= 0 || len > max_pos) {  // no position (a padded sequence), or one that the cache does not have
        if (len != 0 && lane == 0) atomicOr(err, kErrRange);
        return;
    }
    __syncthreads();
    uint8_t *block = cache + ((size_t(t) * n_kv + (j - n_heads)) * (max_pos / kPos) + p / kPos) * block_bytes(d);
    const int q = p % kPos;
    if (lane < d / 8) {
        const Quantised zv = quantise8(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = row_sh[8 * lane + e];
        const Quantised zk = quantise8(x);
        store_key<NG>(block, q, lane, zk);
        if ((lane & 7) == 0) store_value_scale<NG>(block, q, lane >> 3, zv);
        code_sh[lane] = zv.word;
        if (zk.bad || zv.bad) atomicOr(err, kErrNonfinite);
    }
    __syncthreads();
    const int c = (q & 15) >> 2, shift = nibble_bit(4 * (q >> 4) + (q & 3));
#pragma unroll
    for (int dim = lane; dim < d; dim += 64) {
        uint32_t *dst = reinterpret_cast<uint32_t *>(block + v_codes(d) + code_offset(dim >> 4, c * 16 + (dim & 15)));
        const uint32_t code = (code_sh[dim >> 3] >> nibble_bit(dim & 7)) & 15u;
        *dst = (*dst & ~(15u << shift)) | (code << shift);
    }
}

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace

bool attention_int4_shape_supported(int H, int n_heads, int n_kv, int d, int max_pos) {
    return H > 0 && H % 128 == 0 && H <= 1 << 24 && n_heads > 0 && n_kv > 0 && n_heads % n_kv == 0 && n_heads <= 1024 &&
           (d == 64 || d == 128 || d == 192 || d == 256) && (n_heads * d) % 128 == 0 && max_pos > 0 &&
           max_pos % kPos == 0 && max_pos <= MOE_KV4_MAX_POS;
}

// (the attention's and the projections' parts share their place: they follow one another)
size_t attention_int4_workspace_bytes(int T, int H, int n_heads, int n_kv, int d, int max_pos) {
    return align256(sizeof(float) * size_t(T) * (n_heads + 2 * n_kv) * d) + align256(sizeof(float) * size_t(T) * n_heads * d) +
           std::max(kv4_attention_workspace_bytes(T, T, n_heads, n_kv, d, 1, max_pos),
                    matvec_int4_workspace_bytes(T, std::max(H, n_heads * d)));
}

hipError_t launch_attention_decode_int4(float *x, int T, int H, int n_heads, int n_kv, int d, const void *w_qkv,
                                        const void *w_o, void *cache, int max_pos, const int32_t *kv_len, float theta,
                                        void *workspace, int *err, hipStream_t s) {
    const int rows = (n_heads + 2 * n_kv) * d;
    char *ws = static_cast<char *>(workspace);
    float *qkv = reinterpret_cast<float *>(ws);
    float *att = reinterpret_cast<float *>(ws += align256(sizeof(float) * size_t(T) * rows));
    void *aws = ws + align256(sizeof(float) * size_t(T) * n_heads * d);
    hipError_t e = launch_matvec_int4(x, w_qkv, T, rows, H, nullptr, qkv, true, aws, s);
    if (e != hipSuccess) return e;
    const dim3 grid(n_heads + n_kv, T);
    auto *c = static_cast<uint8_t *>(cache);
    switch (d) {
    case 64: heads_kernel<1><<<grid, 64, 0, s>>>(qkv, n_heads, n_kv, theta, kv_len, max_pos, c, err); break;
    case 128: heads_kernel<2><<<grid, 64, 0, s>>>(qkv, n_heads, n_kv, theta, kv_len, max_pos, c, err); break;
    case 192: heads_kernel<3><<<grid, 64, 0, s>>>(qkv, n_heads, n_kv, theta, kv_len, max_pos, c, err); break;
    case 256: heads_kernel<4><<<grid, 64, 0, s>>>(qkv, n_heads, n_kv, theta, kv_len, max_pos, c, err); break;
    default: return hipErrorInvalidValue;
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const Batch batch{nullptr, kv_len, T, T, 1, max_pos};
    e = launch_kv4_attention(qkv, MOE_F32, rows, cache, batch, n_heads, n_kv, d, 0, 1.f / sqrtf(float(d)), att,
                             (long long)n_heads * d, aws, err, s);
    if (e != hipSuccess) return e;
    return launch_matvec_int4(att, w_o, T, H, n_heads * d, x, x, false, aws, s);
}

}  // namespace moe
