// kv4_store.hip -- keys and values quantised to 4 bits as they are written into the cache, and read back.
//
// The bound is bytes: 4 d (bf16) read and 1.125 d written per position and head.  A block of threads takes one
// 32-position block of one head: 8 lanes hold a group of 64 dims, find its range and form its codes.  A key's
// word belongs to one position, a value's word to 8 positions of one dim: the values' codes are turned through
// LDS, and a word that only some of the new positions cover keeps the others' nibbles (read, merged, written
// by the one lane that owns it).
#include "device_common.h"
#include "internal.h"
#include "kv4.h"

namespace moe {
namespace {

using namespace kv4;

// 8 consecutive elements of a row (16-byte aligned).
template <bool F32>
__device__ __forceinline__ void load8(const void *p, size_t i, float (&x)[8]) {
    if constexpr (F32) {
        const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
        const float4 a = dev::load_f4(q), b = dev::load_f4(q + 1);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint4 a = dev::load16(reinterpret_cast<const uint8_t *>(static_cast<const uint16_t *>(p) + i));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
}

template <bool F32>
__device__ __forceinline__ void store8(void *p, size_t i, const float (&x)[8]) {
    if constexpr (F32) {
        float4 *q = reinterpret_cast<float4 *>(static_cast<float *>(p) + i);
        q[0] = make_float4(x[0], x[1], x[2], x[3]);
        q[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = bf16_rne(x[2 * e]) | (bf16_rne(x[2 * e + 1]) << 16);
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

constexpr int kStoreBlock = 256;

// grid: (blocks of positions that a sequence's new tokens can touch, head, sequence)
template <int NG, bool F32>
__global__ __launch_bounds__(kStoreBlock) void kv4_append_kernel(const void *__restrict__ k, const void *__restrict__ v,
                                                                 long long k_stride, long long v_stride, Batch batch,
                                                                 uint8_t *__restrict__ cache, int *err) {
    constexpr int d = NG * kGroup, NC = d / 8;  // chunks of 8 dims
    __shared__ uint32_t codes[kPos][NC + 1];
    const Seq s = sequence(batch, blockIdx.z);
    const int h = blockIdx.y, n_kv = gridDim.y;
    if (s.bad && blockIdx.x == 0 && h == 0 && threadIdx.x == 0) atomicOr(err, kErrRange);
    const int first = max(s.len - s.n, 0), blk = first / kPos + blockIdx.x;  // (tokens before position 0 are padding)
    if (s.n == 0 || blk * kPos >= s.len) return;
    uint8_t *block = cache + (size_t(blockIdx.z) * n_kv + h) * (batch.max_pos / kPos) * block_bytes(d) +
                     size_t(blk) * block_bytes(d);
    const int p_lo = max(first - blk * kPos, 0), p_hi = min(s.len - blk * kPos, kPos);  // new positions of the block
    const long long t_of_0 = (long long)s.t0 + blk * kPos - (s.len - s.n);              // token of the block's position 0
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPos * NC / kStoreBlock; ++i) {
        const int item = i * kStoreBlock + threadIdx.x, p = item / NC, chunk = item % NC;
        if (p < p_lo || p >= p_hi) continue;  // (the 8 lanes of a group share p)
        float x[8];
        load8<F32>(k, size_t(t_of_0 + p) * k_stride + size_t(h) * d + 8 * chunk, x);
        const Quantised zk = quantise8(x);
        store_key<NG>(block, p, chunk, zk);
        load8<F32>(v, size_t(t_of_0 + p) * v_stride + size_t(h) * d + 8 * chunk, x);
        const Quantised zv = quantise8(x);
        codes[p][chunk] = zv.word;
        if ((chunk & 7) == 0) store_value_scale<NG>(block, p, chunk >> 3, zv);
        bad |= zk.bad || zv.bad;
    }
    if (bad) atomicOr(err, kErrNonfinite);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4 * d / kStoreBlock; ++i) {
        const int item = i * kStoreBlock + threadIdx.x;  // (piece, lane, word of the lane's 16 bytes)
        const int w = (item >> 8) * 4 + (item & 3), lane = (item >> 2) & 63, c = lane >> 4;
        const int dim = 16 * w + (lane & 15), shift = nibble_bit(dim & 7);
        uint32_t word = 0, keep = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = 16 * (e >> 2) + 4 * c + (e & 3);
            if (p >= p_lo && p < p_hi) word |= ((codes[p][dim >> 3] >> shift) & 15u) << nibble_bit(e);
            else keep |= 15u << nibble_bit(e);
        }
        uint32_t *dst = reinterpret_cast<uint32_t *>(block + v_codes(d) + 4 * item);
        if (keep == ~0u) continue;
        *dst = keep ? (*dst & keep) | word : word;
    }
}

// grid: (blocks of positions, head, sequence): the values of the sequence's last n positions, as held.
template <int NG, bool F32>
__global__ __launch_bounds__(kStoreBlock) void kv4_read_kernel(const uint8_t *__restrict__ cache, Batch batch,
                                                               void *__restrict__ k, void *__restrict__ v,
                                                               long long k_stride, long long v_stride, int *err) {
    constexpr int d = NG * kGroup, NC = d / 8;
    const Seq s = sequence(batch, blockIdx.z);
    const int h = blockIdx.y, n_kv = gridDim.y;
    if (s.bad && blockIdx.x == 0 && h == 0 && threadIdx.x == 0) atomicOr(err, kErrRange);
    // blocks of positions from the first token's, which may lie before position 0 (those rows are zeros)
    const int first = s.len - s.n, b0 = first >= 0 ? first / kPos : -((-first + kPos - 1) / kPos);
    const int blk = b0 + blockIdx.x;
    if (s.n == 0 || blk * kPos >= s.len) return;
    const uint8_t *block = cache + (size_t(blockIdx.z) * n_kv + h) * (batch.max_pos / kPos) * block_bytes(d) +
                           size_t(max(blk, 0)) * block_bytes(d);
    const int p_lo = max(first - blk * kPos, 0), p_hi = min(s.len - blk * kPos, kPos);
    const long long t_of_0 = (long long)s.t0 + blk * kPos - first;
#pragma unroll 1
    for (int i = 0; i < kPos * NC / kStoreBlock; ++i) {
        const int item = i * kStoreBlock + threadIdx.x, p = item / NC, chunk = item % NC, g = chunk >> 3;
        if (p < p_lo || p >= p_hi) continue;
        float x[8], y[8];
        if (blk < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
        } else {
            const int o = g * kPos + order_index(p), n = p & 15, tile = p >> 4;
            const uint32_t kw = *reinterpret_cast<const uint32_t *>(
                block + k_codes(d) + code_offset(tile * 2 * NG + (chunk >> 2), (chunk & 3) * 16 + n));
            const float ks = bf16_float(reinterpret_cast<const uint16_t *>(block + k_scales(d))[o]);
            const float km = bf16_float(reinterpret_cast<const uint16_t *>(block + k_bases(d))[g * kPos + 2 * n + tile]);
            const float vs = bf16_float(reinterpret_cast<const uint16_t *>(block + v_scales(d))[o]);
            const float vm = bf16_float(reinterpret_cast<const uint16_t *>(block + v_bases(d))[o]);
            const int c = n >> 2, shift = nibble_bit(4 * tile + (n & 3));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int dim = 8 * chunk + e;
                const uint32_t vw = *reinterpret_cast<const uint32_t *>(block + v_codes(d) +
                                                                        code_offset(dim >> 4, c * 16 + (dim & 15)));
                x[e] = fmaf(float((kw >> nibble_bit(e)) & 15u), ks, km);
                y[e] = fmaf(float((vw >> shift) & 15u), vs, vm);
            }
        }
        if (k) store8<F32>(k, size_t(t_of_0 + p) * k_stride + size_t(h) * d + 8 * chunk, x);
        if (v) store8<F32>(v, size_t(t_of_0 + p) * v_stride + size_t(h) * d + 8 * chunk, y);
    }
}

}  // namespace

hipError_t launch_kv4_append(const void *k, const void *v, int dtype, long long k_stride, long long v_stride,
                             const kv4::Batch &batch, int n_kv, int d, void *cache, int *err, hipStream_t s) {
    const dim3 grid((batch.max_q + 2 * kPos - 2) / kPos, n_kv, batch.n_seq);
    auto *c = static_cast<uint8_t *>(cache);
#define KV4_APPEND(NG)                                                                                          \
    case NG * kGroup:                                                                                           \
        if (dtype == MOE_F32) kv4_append_kernel<NG, true><<<grid, kStoreBlock, 0, s>>>(k, v, k_stride, v_stride, batch, c, err); \
        else kv4_append_kernel<NG, false><<<grid, kStoreBlock, 0, s>>>(k, v, k_stride, v_stride, batch, c, err); \
        break;
    switch (d) {
        KV4_APPEND(1) KV4_APPEND(2) KV4_APPEND(3) KV4_APPEND(4)
    default: return hipErrorInvalidValue;
    }
#undef KV4_APPEND
    return hipGetLastError();
}

hipError_t launch_kv4_read(const void *cache, const kv4::Batch &batch, int n_kv, int d, void *k, void *v, int dtype,
                           long long k_stride, long long v_stride, int *err, hipStream_t s) {
    const dim3 grid((batch.max_q + 2 * kPos - 2) / kPos, n_kv, batch.n_seq);
    auto *c = static_cast<const uint8_t *>(cache);
#define KV4_READ(NG)                                                                                            \
    case NG * kGroup:                                                                                           \
        if (dtype == MOE_F32) kv4_read_kernel<NG, true><<<grid, kStoreBlock, 0, s>>>(c, batch, k, v, k_stride, v_stride, err); \
        else kv4_read_kernel<NG, false><<<grid, kStoreBlock, 0, s>>>(c, batch, k, v, k_stride, v_stride, err);  \
        break;
    switch (d) {
        KV4_READ(1) KV4_READ(2) KV4_READ(3) KV4_READ(4)
    default: return hipErrorInvalidValue;
    }
#undef KV4_READ
    return hipGetLastError();
}

}  // namespace moe
