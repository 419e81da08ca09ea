// paged_store.hip -- a paged cache's tables, its store, and the masks of drafted trees.
#include "attend_common.h"
#include "device_common.h"
#include "internal.h"
#include "paged.h"

#include <algorithm>

namespace moe {
namespace {

using namespace paged;

// ---- tables ----------------------------------------------------------------------------------------------------
//
// A prefix sum over the sequences' tokens and one over the pages they need, then a search per page and per token.
// One block does that: the bytes are few (a microsecond's worth at a copy's rate at most), so what counts is one launch
// and its chain of loads, scans and searches (5.7 us for 256 sequences of one token each); the rows of many tokens are a
// launch of their own.
constexpr int kTabBlock = 1024, kTabPer = 2, kTabSeqs = kTabBlock * kTabPer;
constexpr uint32_t kTabCap = 1u << 30;  // sums end there (it is past any row or page there is)

__device__ __forceinline__ uint32_t capped(uint32_t a, uint32_t b) { return min(a + b, kTabCap); }

// Capped sums of v over the block's threads in front of this one; `total` over all.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *sums, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = v;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t o = __shfl_up(upto, k);
        if (lane >= k) upto = capped(upto, o);
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kTabBlock / 64; ++w) {
        const uint32_t s = sums[w];
        if (w < wave) before = capped(before, s);
        total = capped(total, s);
    }
    __syncthreads();
    const uint32_t own = __shfl_up(upto, 1);
    return lane ? capped(before, own) : before;
}

// Whether position `pos` lies on a page that its sequence had before the step (with `len` positions): the one that it
// continues.  Such a page that is missing is an error of its own; what this step's list lacked or held wrong has been reported.
__device__ __forceinline__ bool on_held_page(int pos, int len, int shift) {
    return (pos >> shift) < ((len + (1 << shift) - 1) >> shift);
}

// The last of `n` ascending starts that is at most x (start[0] <= x).
__device__ __forceinline__ int owner(const uint32_t *start, int n, uint32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ROWS: the tokens' rows too.
template <bool ROWS>
__global__ __launch_bounds__(kTabBlock) void page_tables_kernel(TableArgs a, int *err) {
    __shared__ uint32_t tok_sh[kTabSeqs], page_sh[kTabSeqs], sums[kTabBlock / 64];
    __shared__ int len_sh[kTabSeqs];
    const int tid = threadIdx.x, page = 1 << a.shift;
    const uint32_t first = a.free_first ? uint32_t(max(*a.free_first, 0)) : 0u;
    const long long most = (long long)a.max_pages << a.shift;
    uint32_t tok0 = 0, page0 = 0;  // tokens and pages of the sequences in front of these
    bool range = a.free_first && (*a.free_first < 0 || *a.free_first > a.n_free), budget = false;
#pragma unroll 1
    for (int base = 0; base < a.n_seq; base += kTabSeqs) {
        const int count = min(kTabSeqs, a.n_seq - base);
        int len[kTabPer], n[kTabPer];
        uint32_t sum = 0, total;
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int b = base + tid * kTabPer + i;
            len[i] = n[i] = 0;
            if (b < a.n_seq) {
                len[i] = a.kv_len[b];
                n[i] = a.n_new ? a.n_new[b] : 1;
                if (len[i] < 0 || len[i] > most) len[i] = n[i] = 0, range = true;
                if (n[i] < 0 || len[i] + (long long)n[i] > most) n[i] = 0, range = true;
            }
            sum = capped(sum, uint32_t(n[i]));
        }
        uint32_t at = capped(tok0, block_scan(sum, sums, total)), need[kTabPer], pages = 0;
        tok0 = capped(tok0, total);
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            // (tokens past the last row are not there)
            const uint32_t start = min(at, uint32_t(a.T)), end = min(capped(at, uint32_t(n[i])), uint32_t(a.T));
            at = capped(at, uint32_t(n[i]));
            if (int(end - start) != n[i]) range = true;
            n[i] = int(end - start);
            need[i] = uint32_t((len[i] + n[i] + page - 1) >> a.shift) - uint32_t((len[i] + page - 1) >> a.shift);
            pages += need[i];
            const int b = tid * kTabPer + i;
            if (b < count) {
                tok_sh[b] = start;
                len_sh[b] = len[i];
                a.q_start[base + b] = int(start);
                a.kv_len_out[base + b] = len[i] + n[i];
            }
        }
        uint32_t rank = capped(page0, block_scan(pages, sums, total));
        const uint32_t page_end = capped(page0, total);
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int b = tid * kTabPer + i;
            if (b < count) page_sh[b] = rank;
            rank = capped(rank, need[i]);
        }
        __syncthreads();
#pragma unroll 1
        for (uint32_t r = page0 + tid; r < page_end; r += kTabBlock) {
            const int b = owner(page_sh, count, r);
            const uint32_t f = first + r;
            int32_t p = -1;
            if (f < uint32_t(a.n_free)) {
                p = a.free_pages[f];
                if (uint32_t(p) >= uint32_t(a.n_pages)) p = -1, range = true;
            } else {
                budget = true;
            }
            a.table[size_t(base + b) * a.max_pages + ((len_sh[b] + page - 1) >> a.shift) + (r - page_sh[b])] = p;
        }
        __syncthreads();
        if constexpr (ROWS) {
            const uint32_t t_end = min(tok0, uint32_t(a.T));
#pragma unroll 1
            for (uint32_t t = tok_sh[0] + tid; t < t_end; t += kTabBlock) {
                const int b = owner(tok_sh, count, t), pos = len_sh[b] + int(t - tok_sh[b]);
                const int32_t p = a.table[size_t(base + b) * a.max_pages + (pos >> a.shift)];
                const bool there = uint32_t(p) < uint32_t(a.n_pages);
                range |= !there && on_held_page(pos, len_sh[b], a.shift);
                if (a.positions) a.positions[t] = pos;
                if (a.slots) a.slots[t] = there ? (p << a.shift) + (pos & (page - 1)) : -1;
            }
            __syncthreads();
        }
        page0 = page_end;
    }
    const uint32_t rows = min(tok0, uint32_t(a.T));
    if constexpr (ROWS)
        for (uint32_t t = rows + tid; t < uint32_t(a.T); t += kTabBlock) {
            if (a.positions) a.positions[t] = -1;
            if (a.slots) a.slots[t] = -1;
        }
    if (tid == 0) {
        a.q_start[a.n_seq] = int(rows);
        if (a.free_next) *a.free_next = int(min(min(first, uint32_t(a.n_free)) + page0, uint32_t(a.n_free)));
    }
    const int bits = (range ? kErrRange : 0) | (budget ? kErrBudget : 0);
    if (bits) atomicOr(err, bits);
}

// The rows of many tokens, behind page_tables_kernel<false>: 1024 of them per block.
constexpr int kRowsBlock = 256, kRowsPer = 4;
__global__ __launch_bounds__(kRowsBlock) void page_rows_kernel(TableArgs a, int *err) {
    __shared__ uint32_t tok_sh[kTabSeqs];
    __shared__ int len_sh[kTabSeqs];
    const int tid = threadIdx.x;
    const uint32_t t0 = blockIdx.x * uint32_t(kRowsBlock * kRowsPer), t1 = min(t0 + kRowsBlock * kRowsPer, uint32_t(a.T));
    const uint32_t rows = uint32_t(a.q_start[a.n_seq]);
    bool range = false;
#pragma unroll 1
    for (int base = 0; base < a.n_seq; base += kTabSeqs) {
        const int count = min(kTabSeqs, a.n_seq - base);
        const uint32_t from = uint32_t(a.q_start[base]), to = uint32_t(a.q_start[base + count]);
        if (to <= t0) continue;
        if (from >= t1) break;
        __syncthreads();
#pragma unroll 4
        for (int b = tid; b < count; b += kRowsBlock) {
            const int start = a.q_start[base + b];
            tok_sh[b] = uint32_t(start);
            len_sh[b] = a.kv_len_out[base + b] - (a.q_start[base + b + 1] - start);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRowsPer; ++i) {
            const uint32_t t = t0 + i * kRowsBlock + tid;
            if (t < from || t >= min(to, t1)) continue;
            const int b = owner(tok_sh, count, t), pos = len_sh[b] + int(t - tok_sh[b]);
            const int32_t p = a.table[size_t(base + b) * a.max_pages + (pos >> a.shift)];
            const bool there = uint32_t(p) < uint32_t(a.n_pages);
            range |= !there && on_held_page(pos, len_sh[b], a.shift);
            if (a.positions) a.positions[t] = pos;
            if (a.slots) a.slots[t] = there ? (p << a.shift) + (pos & ((1 << a.shift) - 1)) : -1;
        }
    }
#pragma unroll
    for (int i = 0; i < kRowsPer; ++i) {
        const uint32_t t = t0 + i * kRowsBlock + tid;
        if (t < rows || t >= t1) continue;
        if (a.positions) a.positions[t] = -1;
        if (a.slots) a.slots[t] = -1;
    }
    if (range) atomicOr(err, kErrRange);
}

// ---- store -----------------------------------------------------------------------------------------------------
constexpr int kStoreBlock = 256, kStoreLaunch = 1 << 22;  // blocks of a launch, at most

// A thread takes 8 dims of a token's head, a block so many tokens that its threads have one such piece each.  Bytes bound it
// (16384 tokens, 8 heads of 128 in bf16, 133 MB read and written: 26.3 us, 5.1 TB/s, a large copy 4.8); of few tokens, the
// launch (2.5 us).  fp32 is rounded once, to nearest, ties to even.  grid: (groups of tokens, keys or values)
template <bool F32>
__global__ __launch_bounds__(kStoreBlock) void paged_append_kernel(const void *k, const void *v, long long k_stride,
                                                                   long long v_stride, int T, int n_kv, int d,
                                                                   const int32_t *slots, Pages pages, int per_block, int *err) {
    const bool values = blockIdx.y;
    const int per = n_kv * (d / 8), local = threadIdx.x / per;
    const int t = int(blockIdx.x) * per_block + local;
    if (local >= per_block || t >= T) return;
    const int slot = slots[t];
    if (slot == -1) return;
    if (slot < 0 || (slot >> pages.shift) >= pages.n_pages) {
        atomicOr(err, kErrRange);
        return;
    }
    uint16_t *dst = (values ? pages.v : pages.k) + (slot >> pages.shift) * (values ? pages.v_stride : pages.k_stride);
    const int off = slot & ((1 << pages.shift) - 1);
#pragma unroll 1
    for (int c = threadIdx.x - local * per; c < per; c += kStoreBlock) {
        const int h = c / (d / 8), i = (c - h * (d / 8)) * 8;
        const size_t at = size_t(t) * (values ? v_stride : k_stride) + size_t(h) * d + i;
        const uint8_t *src = static_cast<const uint8_t *>(values ? v : k) + at * (F32 ? 4 : 2);
        uint4 w = dev::load16(src);
        if constexpr (F32) {
            const uint4 u = dev::load16(src + 16);
            auto pack = [](uint32_t lo, uint32_t hi) { return attend::pack_bf16(__uint_as_float(lo), __uint_as_float(hi)); };
            w = make_uint4(pack(w.x, w.y), pack(w.z, w.w), pack(u.x, u.y), pack(u.z, u.w));
        }
        *reinterpret_cast<uint4 *>(dst + ((size_t(h) << pages.shift) + off) * d + i) = w;
    }
}

// ---- trees -----------------------------------------------------------------------------------------------------
//
// A token's bits are its own and its parent's: with every round a token takes over those of the token that its chain has
// reached and doubles the chain, so that a depth of 256 takes 8 rounds.  The rounds' latency is what it takes (16 trees of 25
// tokens 5.3 us, one of 60 3.6).  grid: sequences
__global__ __launch_bounds__(MOE_MAX_TREE) void tree_masks_kernel(const int32_t *parents, kv4::Batch batch, int words,
                                                                  unsigned long long *masks, int32_t *positions, int *err) {
    constexpr int W = MOE_MAX_TREE / 64;
    __shared__ unsigned long long mask_sh[W][MOE_MAX_TREE];
    __shared__ int up_sh[MOE_MAX_TREE];
    const int b = blockIdx.x, i = threadIdx.x;
    int t0 = batch.q_start ? batch.q_start[b] : b, end = batch.q_start ? batch.q_start[b + 1] : b + 1;
    bool bad = t0 < 0 || end < t0 || end > batch.T || end - t0 > batch.max_q;
    const int n = bad ? 0 : end - t0;
    int len = n;
    if (batch.kv_len) {
        len = batch.kv_len[b];
        if (len < 0) len = 0, bad = true;
    }
    int up = -1;
    if (i < n) {
        up = parents[t0 + i];
        if (up < -1 || up >= i) up = -1, bad = true;
    }
    unsigned long long m[W];
#pragma unroll
    for (int w = 0; w < W; ++w) mask_sh[w][i] = m[w] = i >> 6 == w ? 1ull << (i & 63) : 0;
    up_sh[i] = up;
    while (__syncthreads_or(up >= 0)) {
        const int next = up >= 0 ? up_sh[up] : -1;
        if (up >= 0)
#pragma unroll
            for (int w = 0; w < W; ++w) m[w] |= mask_sh[w][up];
        __syncthreads();
        up_sh[i] = up = next;
#pragma unroll
        for (int w = 0; w < W; ++w) mask_sh[w][i] = m[w];
    }
    if (bad) atomicOr(err, kErrRange);
    if (i >= n) return;
    int bits = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        bits += __popcll(m[w]);
        if (w < words) masks[size_t(t0 + i) * words + w] = m[w];
    }
    if (positions) positions[t0 + i] = len - n - 1 + bits;
}

}  // namespace

hipError_t launch_page_tables(const paged::TableArgs &a, int *err, hipStream_t s) {
    // One launch up to 8192 rows (16 sequences, 5000 rows in all: 9.3 us a call, 11.6 with a second launch for the rows; 10000:
    // 10.7 and 11.5; 61 prompts, 60000: 41 and 11.7).
    if (a.T <= 8192) {
        page_tables_kernel<true><<<1, kTabBlock, 0, s>>>(a, err);
    } else {
        page_tables_kernel<false><<<1, kTabBlock, 0, s>>>(a, err);
        page_rows_kernel<<<(a.T + kRowsBlock * kRowsPer - 1) / (kRowsBlock * kRowsPer), kRowsBlock, 0, s>>>(a, err);
    }
    return hipGetLastError();
}

hipError_t launch_paged_append(const void *k, const void *v, int dtype, long long k_stride, long long v_stride, int T,
                               int n_kv, int d, const int32_t *slots, const paged::Pages &pages, int *err, hipStream_t s) {
    const int per_block = std::max(1, kStoreBlock / (n_kv * (d / 8)));
    // A launch has fewer than 2^32 threads.
    const int most = kStoreLaunch * per_block;
    const size_t size = dtype == MOE_F32 ? 4 : 2;
    for (int t0 = 0; t0 < T; t0 += most) {
        const int count = std::min(T - t0, most);
        const dim3 grid((count + per_block - 1) / per_block, 2);
        const uint8_t *k0 = static_cast<const uint8_t *>(k) + t0 * k_stride * size, *v0 = static_cast<const uint8_t *>(v) + t0 * v_stride * size;
        const auto kernel = dtype == MOE_F32 ? paged_append_kernel<true> : paged_append_kernel<false>;
        kernel<<<grid, kStoreBlock, 0, s>>>(k0, v0, k_stride, v_stride, count, n_kv, d, slots + t0, pages, per_block, err);
    }
    return hipGetLastError();
}

hipError_t launch_tree_masks(const int32_t *parents, const kv4::Batch &batch, int words, uint64_t *masks, int32_t *positions,
                             int *err, hipStream_t s) {
    tree_masks_kernel<<<batch.n_seq, MOE_MAX_TREE, 0, s>>>(parents, batch, words, reinterpret_cast<unsigned long long *>(masks),
                                                           positions, err);
    return hipGetLastError();
}

}  // namespace moe
