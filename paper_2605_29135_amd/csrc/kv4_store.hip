// kv4_store.hip -- keys and values quantised to 4 bits as they are written into the cache, and read back.
//
// The bound is bytes: 4 d (bf16) read and 1.125 d written per position and head.  A block of threads takes one
// 32-position block of one head: 8 lanes hold a group of 64 dims, find its range and form its codes.  A key's
// word belongs to one position, a value's word to 8 positions of one dim: the values' codes are turned through
// LDS, and a word that only some of the new positions cover keeps the others' nibbles (read ahead, merged, written
// by the one lane that owns it).  Everything is written from LDS in the cache's order, in whole lines.
//
// Measured (8 heads of 128, bf16): 6 311 new positions of four sequences 13.7 us (33 MB, 2.4 TB/s), read back 9.6 us
// (3.4 TB/s); one new position of 16 sequences 4.4 and 3.1 us, which is a launch and its chain of loads.  The long form's
// bytes are 6.5 us at a copy's rate, and the lanes issue for 7.6 us of the append (23 operations per element, counted) and
// 3.3 of the read: the device holds all of the blocks that have work at once, they load, then compute, then store
// together, and little of the one runs under the other.  (Blocks beyond a sequence's tokens cost 0.5 us of the read, and
// none of the append: 199 per sequence and head were launched, 65 would do.  Written straight to the cache, a nibble's word
// at a time, the append took 21 us.)
#include "device_common.h"
#include "internal.h"
#include "kv4.h"

namespace moe {
namespace {

using namespace kv4;

// 8 consecutive elements of a row (16-byte aligned), as they lie and in fp32.
template <bool F32>
struct Eight {
    uint4 raw[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void *p, size_t i) {
        const uint8_t *q = static_cast<const uint8_t *>(p) + i * (F32 ? 4 : 2);
#pragma unroll
        for (int e = 0; e < (F32 ? 2 : 1); ++e) raw[e] = dev::load16(q + 16 * e);
    }
    __device__ __forceinline__ void floats(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < (F32 ? 2 : 1); ++e) {
            const uint32_t w[4] = {raw[e].x, raw[e].y, raw[e].z, raw[e].w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if constexpr (F32) x[4 * e + u] = __uint_as_float(w[u]);
                else {
                    x[2 * u] = __uint_as_float(w[u] << 16);
                    x[2 * u + 1] = __uint_as_float(w[u] & 0xffff0000u);
                }
            }
        }
    }
};

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

// Position (of 32) of entry i of a scale or base array: the order 8 c + i, or for the keys' bases [position][tile].
__device__ __forceinline__ int entry_position(int i, bool tiles) {
    return tiles ? 16 * (i & 1) + (i >> 1) : 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3);
}

// grid: (blocks of positions that a sequence's new tokens can touch, head, sequence)
template <int NG, bool F32>
__global__ __launch_bounds__(kStoreBlock) void kv4_append_kernel(const void *__restrict__ k, const void *__restrict__ v,
                                                                 long long k_stride, long long v_stride, Batch batch,
                                                                 uint8_t *__restrict__ cache, int *err) {
    constexpr int d = NG * kGroup, NC = d / 8, R = kPos * NC / kStoreBlock;  // chunks of 8 dims; items per thread
    __shared__ uint32_t codes[2][kPos][NC + 1], params[2][NG][kPos];         // of keys and values; scale and base
    const Seq s = sequence(batch, blockIdx.z);
    const int h = blockIdx.y, n_kv = gridDim.y, tid = threadIdx.x;
    if (s.bad && blockIdx.x == 0 && h == 0 && tid == 0) atomicOr(err, kErrRange);
    const int first = max(s.len - s.n, 0), blk = first / kPos + blockIdx.x;  // (tokens before position 0 are padding)
    if (s.n == 0 || blk * kPos >= s.len) return;
    uint8_t *block = cache + (size_t(blockIdx.z) * n_kv + h) * (batch.max_pos / kPos) * block_bytes(d) +
                     size_t(blk) * block_bytes(d);
    const int p_lo = max(first - blk * kPos, 0), p_hi = min(s.len - blk * kPos, kPos);  // new positions of the block
    const long long t_of_0 = (long long)s.t0 + blk * kPos - (s.len - s.n);              // token of the block's position 0
    // A thread's words of the codes: consecutive ones of the piece-wise arrays (4 d of keys, 4 d of values).
    uint32_t *kw = reinterpret_cast<uint32_t *>(block + k_codes(d)), *vw = reinterpret_cast<uint32_t *>(block + v_codes(d));
    const bool whole = p_lo == 0 && p_hi == kPos;
    uint32_t old[R];
    if (!whole)
#pragma unroll
        for (int i = 0; i < R; ++i) old[i] = vw[i * kStoreBlock + tid];
    // (all the loads before any use: a position that is not new reads the nearest one that is)
    Eight<F32> ek[R], ev[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int item = i * kStoreBlock + tid, chunk = item % NC;
        const size_t token = size_t(t_of_0 + min(max(item / NC, p_lo), p_hi - 1));
        ek[i].load(k, token * k_stride + size_t(h) * d + 8 * chunk);
        ev[i].load(v, token * v_stride + size_t(h) * d + 8 * chunk);
    }
    __builtin_amdgcn_sched_barrier(0);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int item = i * kStoreBlock + tid, p = item / NC, chunk = item % NC;
        if (p < p_lo || p >= p_hi) continue;  // (the 8 lanes of a group share p)
        float x[8], y[8];
        ek[i].floats(x);
        ev[i].floats(y);
        const Quantised zk = quantise8(x), zv = quantise8(y);
        codes[0][p][chunk] = zk.word;
        codes[1][p][chunk] = zv.word;
        if ((chunk & 7) == 0) {
            params[0][chunk >> 3][p] = zk.s | (uint32_t(zk.m) << 16);
            params[1][chunk >> 3][p] = zv.s | (uint32_t(zv.m) << 16);
        }
        bad |= zk.bad || zv.bad;
    }
    if (bad) atomicOr(err, kErrNonfinite);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int item = i * kStoreBlock + tid;  // (piece, lane, word of the lane's 16 bytes)
        const int w = (item >> 8) * 4 + (item & 3), lane = (item >> 2) & 63, c = lane >> 4, n = lane & 15;
        const int p = 16 * (w / (2 * NG)) + n;
        if (p >= p_lo && p < p_hi) kw[item] = codes[0][p][4 * (w % (2 * NG)) + c];
        const int dim = 16 * w + n, shift = nibble_bit(dim & 7);
        uint32_t word = 0, keep = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int q = 16 * (e >> 2) + 4 * c + (e & 3);
            if (whole || (q >= p_lo && q < p_hi)) word |= ((codes[1][q][dim >> 3] >> shift) & 15u) << nibble_bit(e);
            else keep |= 15u << nibble_bit(e);
        }
        if (whole) vw[item] = word;
        else if (keep != ~0u) vw[item] = (old[i] & keep) | word;
    }
#pragma unroll
    for (int i = tid; i < 4 * NG * kPos; i += kStoreBlock) {  // arrays of scales and bases, keys' then values'
        const int array = i / (NG * kPos), p = entry_position(i % kPos, array == 1);
        if (p < p_lo || p >= p_hi) continue;
        const uint32_t sm = params[array >> 1][(i / kPos) % NG][p];
        reinterpret_cast<uint16_t *>(block + k_scales(d))[i] = uint16_t(array & 1 ? sm >> 16 : sm);
    }
}

// grid: (blocks of positions, head, sequence): the values of the sequence's last n positions, as held.  A block goes
// through LDS as it lies; 8 lanes form 64 dims of a position.
template <int NG, bool F32>
__global__ __launch_bounds__(kStoreBlock) void kv4_read_kernel(const uint8_t *__restrict__ cache, Batch batch,
                                                               void *__restrict__ k, void *__restrict__ v,
                                                               long long k_stride, long long v_stride, int *err) {
    constexpr int d = NG * kGroup, NC = d / 8, R = kPos * NC / kStoreBlock;
    __shared__ uint4 held[block_bytes(d) / 16];
    const Seq s = sequence(batch, blockIdx.z);
    const int h = blockIdx.y, n_kv = gridDim.y, tid = threadIdx.x;
    if (s.bad && blockIdx.x == 0 && h == 0 && tid == 0) atomicOr(err, kErrRange);
    // blocks of positions from the first token's, which may lie before position 0 (those rows are zeros)
    const int first = s.len - s.n, b0 = first >= 0 ? first / kPos : -((-first + kPos - 1) / kPos);
    const int blk = b0 + blockIdx.x;
    if (s.n == 0 || blk * kPos >= s.len) return;
    const int p_lo = max(first - blk * kPos, 0), p_hi = min(s.len - blk * kPos, kPos);
    const long long t_of_0 = (long long)s.t0 + blk * kPos - first;
    if (blk >= 0) {
        const uint8_t *block = cache + (size_t(blockIdx.z) * n_kv + h) * (batch.max_pos / kPos) * block_bytes(d) +
                               size_t(blk) * block_bytes(d);
#pragma unroll
        for (int i = 0; i < int((block_bytes(d) / 16 + kStoreBlock - 1) / kStoreBlock); ++i)
            if (i * kStoreBlock + tid < int(block_bytes(d) / 16))
                held[i * kStoreBlock + tid] = dev::load16(block + (i * kStoreBlock + tid) * 16);
    }
    __syncthreads();
    const uint8_t *block = reinterpret_cast<const uint8_t *>(held);
#pragma unroll 2
    for (int i = 0; i < R; ++i) {
        const int item = i * kStoreBlock + tid, p = item / NC, chunk = item % NC, g = chunk >> 3;
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
