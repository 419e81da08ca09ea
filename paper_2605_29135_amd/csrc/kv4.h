// kv4.h -- layout of the 4-bit key/value cache, shared by the kernels that write, read and attend over it.
//
// A head vector of d = 64 NG dims is held as 4-bit codes with a scale s and a base m (bf16) per group of 64
// dims: value = s u + m.  One sequence and key/value head is a run of blocks of 32 positions, 36 d bytes each:
//   K codes 16 d | V codes 16 d | K scales d | K bases d | V scales d | V bases d.
// The order inside is that of the operands of the 16x16x32 matrix product (lane l: row or column n = l % 16,
// elements k = 8 c + i, c = l / 16, i < 8), so that a lane loads its operands 16 bytes at a time and nothing
// is moved between lanes:
//   K codes: word w = tile * 2 NG + j of lane l holds dims 32 j + 8 c + i of position 16 tile + n; word w is
//            word w % 4 of the lane's 16 bytes in the 1 KiB piece w / 4;
//   V codes: word t of lane l holds dim 16 t + n of the positions order(8 c + i), pieces as above;
//   K scales, V scales, V bases: [NG][32 positions in the order 8 c + i];
//   K bases: [NG][16 positions][2 tiles].
// order(8 c + i) = 16 (i / 4) + 4 c + i % 4: the positions whose scores lane (n, c) holds after the score
// products of the block's two tiles, which therefore are its operand of the value product as they stand.
// Element i of a word is its nibble i / 2 + 4 (i % 2): one shift and one bit operation give two operands.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moe {
namespace kv4 {

constexpr int kGroup = 64;  // dims per scale and base
constexpr int kPos = 32;    // positions per block

__host__ __device__ constexpr size_t block_bytes(int d) { return size_t(36) * d; }
__host__ __device__ constexpr int k_codes(int) { return 0; }
__host__ __device__ constexpr int v_codes(int d) { return 16 * d; }
__host__ __device__ constexpr int k_scales(int d) { return 32 * d; }
__host__ __device__ constexpr int k_bases(int d) { return 33 * d; }
__host__ __device__ constexpr int v_scales(int d) { return 34 * d; }
__host__ __device__ constexpr int v_bases(int d) { return 35 * d; }

// Byte offset of word w of lane l in a piece-wise array of codes.
__device__ __forceinline__ int code_offset(int w, int lane) { return ((w >> 2) * 64 + lane) * 16 + (w & 3) * 4; }
// Index of position p (of 32) in the order 8 c + i.
__device__ __forceinline__ int order_index(int p) { return 8 * ((p & 15) >> 2) + 4 * (p >> 4) + (p & 3); }
// Bit of element i of a word.
__device__ __forceinline__ int nibble_bit(int i) { return 4 * ((i >> 1) + 4 * (i & 1)); }

// A batch of sequences in a flat list of T tokens: sequence b's tokens are q_start[b] .. q_start[b + 1) (one
// each without q_start) and lie at the last positions of its kv_len[b].  A sequence whose token range does
// not fit has none here, one whose length does not fit the cache is an empty one; `bad` says so.
struct Batch {
    const int32_t *q_start;  // device [n_seq + 1], or NULL
    const int32_t *kv_len;   // device [n_seq]
    int T, n_seq, max_q, max_pos;
};

struct Seq {
    int t0, n, len;  // first token, tokens, positions
    bool bad;
};

__device__ __forceinline__ Seq sequence(const Batch &b, int i) {
    Seq s;
    s.t0 = b.q_start ? b.q_start[i] : i;
    const int end = b.q_start ? b.q_start[i + 1] : i + 1;
    s.len = b.kv_len[i];
    const bool tokens = s.t0 >= 0 && end >= s.t0 && end <= b.T && end - s.t0 <= b.max_q;
    const bool length = s.len >= 0 && s.len <= b.max_pos;
    s.n = tokens ? end - s.t0 : 0;
    if (!length) s.len = 0;
    s.bad = !tokens || !length;
    return s;
}

// Scale and base (as bf16 bits) and the codes of 8 dims of a group that 8 neighbouring lanes hold, one word
// in the order of nibble_bit.  m = bf16(min), s = bf16((max - m) / 15) with the division as a product by
// fp32(1/15), u = nearest integer to (x - m) / s, ties to even, within 0..15, where x - m is an fp32
// difference.  A group with an element, scale or base that is not finite comes out as zeros, `bad` set.
struct Quantised {
    uint32_t word;
    uint16_t s, m;
    bool bad;
};

__device__ __forceinline__ uint32_t bf16_rne(float f) {
    const uint32_t u = __float_as_uint(f);
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}
__device__ __forceinline__ float bf16_float(uint32_t b) { return __uint_as_float(b << 16); }

template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
template <typename F>
__device__ __forceinline__ float over8(float v, F f) {
    v = f(v, lane_swap<0xB1>(v));   // xor 1
    v = f(v, lane_swap<0x4E>(v));   // xor 2
    return f(v, lane_swap<0x141>(v));  // half-row mirror
}

__device__ __forceinline__ Quantised quantise8(const float (&x)[8]) {
    float lo = x[0], hi = x[0], nan = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        nan = fmaf(x[i], 0.f, nan);  // (an infinity or NaN makes it NaN)
    }
    lo = over8(lo, [](float a, float b) { return fminf(a, b); });
    hi = over8(hi, [](float a, float b) { return fmaxf(a, b); });
    nan = over8(nan, [](float a, float b) { return a + b; });
    Quantised r;
    uint32_t mb = bf16_rne(lo);
    const float m = bf16_float(mb);
    uint32_t sb = bf16_rne((hi - m) * (1.0f / 15.0f));
    r.bad = !(nan == 0.f) || (mb & 0x7f80u) == 0x7f80u || (sb & 0x7f80u) == 0x7f80u;
    // (hi >= m up to the rounding of m: a range below zero, like one below 2^-126, has the scale 0)
    if (r.bad || (sb & 0x8000u) || (sb & 0x7f80u) == 0) sb = 0;
    if (r.bad) mb = 0;
    r.s = uint16_t(sb);
    r.m = uint16_t(mb);
    r.word = 0;
    if (sb) {
        // The quotient by the reciprocal, corrected by its exact remainder, is the nearest fp32 number: k + 1/2 comes
        // out where t / s is that, and nowhere else ((k + 1/2) s has at most 13 bits, so another t is off by 2^-24 of
        // itself, more than half a last place of the quotient).  Adding 2^23 rounds to the nearest integer, ties to
        // even, in the low bits; what the eight sums carry above them goes off at the end.
        const float s = bf16_float(sb), inv = __builtin_amdgcn_rcpf(s);
        uint32_t carry = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = x[i] - m, q0 = t * inv, q = fmaf(fmaf(-q0, s, t), inv, q0);
            r.word += __float_as_uint(__builtin_amdgcn_fmed3f(q, 0.f, 15.f) + 8388608.f) << nibble_bit(i);
            carry += 0x4B000000u << nibble_bit(i);
        }
        r.word -= carry;
    }
    return r;
}

// Stores the codes, scale and base of 8 dims (chunk of 8 within the head) of a key at position p of a block.
// Every lane of a group of 8 calls it with the same p; the first stores the group's scale and base.
template <int NG>
__device__ __forceinline__ void store_key(uint8_t *block, int p, int chunk, const Quantised &z) {
    constexpr int d = NG * kGroup;
    const int tile = p >> 4, n = p & 15;
    *reinterpret_cast<uint32_t *>(block + k_codes(d) + code_offset(tile * 2 * NG + (chunk >> 2), (chunk & 3) * 16 + n)) =
        z.word;
    if ((chunk & 7) == 0) {
        const int g = chunk >> 3;
        reinterpret_cast<uint16_t *>(block + k_scales(d))[g * kPos + order_index(p)] = z.s;
        reinterpret_cast<uint16_t *>(block + k_bases(d))[g * kPos + 2 * n + tile] = z.m;
    }
}
template <int NG>
__device__ __forceinline__ void store_value_scale(uint8_t *block, int p, int g, const Quantised &z) {
    constexpr int d = NG * kGroup;
    reinterpret_cast<uint16_t *>(block + v_scales(d))[g * kPos + order_index(p)] = z.s;
    reinterpret_cast<uint16_t *>(block + v_bases(d))[g * kPos + order_index(p)] = z.m;
}

}  // namespace kv4
}  // namespace moe
