// paged_attention.hip -- attention over a paged bf16 cache: one or many tokens per sequence, a window with first positions
// that stay visible, trees of drafted tokens.
//
// Scores are formed transposed (positions x rows) by the 16x16x32 matrix product, so that a lane holds one row's
// probabilities of the positions that are its operand of the value product (they stay in registers), and the outputs as
// dims x rows, so that a row's running maximum and sum belong to its lane.  The value product wants eight positions of
// one dim in a lane, the cache has eight dims of a position in a row: a lane loads the same dims of eight positions and
// turns them in registers, one operation per pair.  Which dim is which row of the product is free: a lane's own eight
// (or four) dims lie in as many products.
//
// Exact products of bf16, sums in fp32.  fp32 queries enter as three bf16 terms (2^-24 of the element), probabilities as
// three (fp32) or two (bf16: 2^-16) of them: where few rows meet the cache the products cost nothing beside its bytes.
//
// A row is a (token, query head of the group) pair; a wave takes NT tiles of 16 rows over every fourth block of 32
// positions, and the block's waves join their (max, sum, output) through LDS.  With few rows the positions are split over
// more blocks (grid), whose partial results a second launch joins.  Blocks of positions that no token of the sequence sees
// (between the first positions and the window) are stepped over: pages for them need not exist.
#include "attend_common.h"
#include "device_common.h"
#include "internal.h"
#include "paged.h"

#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

using namespace attend;
using namespace paged;

constexpr int kPos = 32;  // positions per block
constexpr int kAttWaves = 4, kAttBlock = 64 * kAttWaves;
// Blocks that fill the device, where rows and heads alone give fewer: two to a unit (32 sequences of up to 16384 positions, 8
// heads of 128: 220 us, 276 with 256, 259 with 384; 64 of up to 2000, 8 heads of 64, of whose blocks four fit: 37 us, 44
// with 1024).
constexpr int kTarget = 512;
// Caches that are never split: the second launch costs more (one token over 500 positions 11.2 us, 13.6 split; three prompts of
// 100 tokens, 300 positions 18.6 and 21.5; 8 tokens over 1500 each 18.4, 17.2 split).
constexpr int kWhole = 512;

struct PagedArgs {
    const void *q;
    void *out;
    Pages pages;
    const int32_t *table;   // [n_seq][max_pages]
    const uint32_t *tree;   // [T][tree_words] bits of the drafted tokens that a token sees, or NULL
    float *part;            // [unit][head][tiles][rows of a tile][d + 4]: unnormalised output, maximum, sum, unit
    long long q_stride, out_stride;
    int max_pages, tree_words;
    int n_kv, group, window, sinks;
    int tiles;              // row tiles of the largest sequence
    float unit;             // from scores to log2 units, positive
    int negate;             // the scale's sign
    Split split;
    int shares;             // 1: the batch may be cut into shares
    Batch batch;
    int *err;
};

// The positions that tokens of a sequence see, as blocks: the first `sink` ones and those from `first` on.
struct Seen {
    int sink, first, count;  // blocks [0, sink) and [first, first + count - sink)
    int from;                // the first position behind the sinks that some token sees
    __device__ __forceinline__ int block(int v) const { return v < sink ? v : v - sink + first; }
};
__device__ __forceinline__ Seen seen(const Seq &s, int window, int sinks) {
    Seen r{0, 0, 0, 0};
    if (s.n == 0 || s.len == 0) return r;
    // (a drafted token stands no earlier than behind the cached ones)
    r.from = window ? max(0, s.len - s.n - window + 1) : 0;
    r.first = r.from / kPos;
    r.sink = min((min(sinks, r.from) + kPos - 1) / kPos, r.first);
    r.count = r.sink + (s.len - 1) / kPos + 1 - r.first;
    return r;
}

// The split of a batch.  Few blocks of positions: sequences are cut into pieces (find_piece).  Many, in the kernel for few
// rows: the blocks of all sequences, one behind the other, are cut into shares for the grid's units, whatever sequences they
// fall into, so that all units have the same to do (of pieces, as many as run together, the longest is a fifth longer than
// the mean: 32 sequences of 4096 to 16384 positions 260 us, shares 220).  A second sequence in a share costs its start, some
// 3 us, so shares have kShare blocks at least (8 sequences of 1024 to 4096: 26 us in pieces, 30 in shares of 10).  A sequence
// with tokens has at least one block, so that its outputs are written.  Every wave works it out for itself.
constexpr int kShare = 32;
__device__ __forceinline__ int blocks_of(const PagedArgs &a, const Seq &s) {
    return s.n ? max(1, seen(s, a.window, a.sinks).count) : 0;
}
struct Spread {
    uint32_t total;  // (a batch that is split has fewer than kTarget sequences of at most 2^21 blocks)
    int chunk;
};
__device__ __forceinline__ Spread spread(const PagedArgs &a, int *err) {
    const int lane = threadIdx.x & 63;
    Spread r{0, 0};
#pragma unroll 1
    for (int base = 0; base < a.batch.n_seq; base += 64) {
        Seq s{0, 0, 0, false};
        if (base + lane < a.batch.n_seq) s = sequence(a.batch, base + lane);
        if (err && s.bad) atomicOr(err, kErrRange);
        r.total += uint32_t(__builtin_amdgcn_readlane(int(wave_scan(uint32_t(blocks_of(a, s)))), 63));
    }
    r.chunk = max(int((r.total + uint32_t(a.split.target) - 1) / uint32_t(a.split.target)), a.split.least);
    return r;
}
// A part of one sequence: its blocks first..end - 1 (counted as in Seen).
struct Share {
    Seq s;
    int seq, first, end;
    int count;  // parts that the sequence has; 0: there is no such one, 1: its outputs are final
    int part;   // number among all parts: those of a sequence follow one another
};
__device__ __forceinline__ Share piece_share(const PagedArgs &a, int want, bool by_unit, int *err) {
    const Piece p = find_piece(a.batch, a.split, [&](const Seq &s) { return seen(s, a.window, a.sinks).count; }, want, by_unit, err);
    return Share{p.s, p.seq, p.split * p.chunk, p.split == p.count - 1 ? 1 << 30 : (p.split + 1) * p.chunk, p.count, p.first + p.split};
}
// This block's piece: grid (row tiles, key/value head, sequence), one each, or with a target (key/value head, row tiles, units).
__device__ __forceinline__ Share this_piece(const PagedArgs &a, int *err) {
    if (a.split.target) return piece_share(a, blockIdx.z, true, blockIdx.z == 0 ? err : nullptr);
    const Share r{sequence(a.batch, blockIdx.z), int(blockIdx.z), 0, 1 << 30, 1, 0};
    if (r.s.bad && err && (threadIdx.x & 63) == 0) atomicOr(err, kErrRange);
    return r;
}
// The share that begins with block g of the batch (below the total) and ends before g_end, or sequence `want`'s first.
__device__ __forceinline__ Share share_at(const PagedArgs &a, int chunk, uint32_t g, uint32_t g_end, int want) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    Share r{};
#pragma unroll 1
    for (int base = 0; base < a.batch.n_seq; base += 64) {
        Seq s{0, 0, 0, false};
        if (base + lane < a.batch.n_seq) s = sequence(a.batch, base + lane);
        const int n = blocks_of(a, s);
        const uint32_t upto = before + wave_scan(uint32_t(n));
        const unsigned long long hit = __ballot(want < 0 ? upto > g : base + lane == want);
        if (hit) {
            const int l = __builtin_amdgcn_readfirstlane(__ffsll(hit) - 1);
            const int blocks = __builtin_amdgcn_readlane(n, l);
            const uint32_t start = uint32_t(__builtin_amdgcn_readlane(int(upto), l)) - uint32_t(blocks);
            if (want >= 0) g = start, g_end = start;
            r.s.t0 = __builtin_amdgcn_readlane(s.t0, l);
            r.s.n = __builtin_amdgcn_readlane(s.n, l);
            r.s.len = __builtin_amdgcn_readlane(s.len, l);
            r.seq = base + l;
            r.first = int(g - start);
            r.end = min(blocks, int(g_end - start));
            const uint32_t unit = start / uint32_t(chunk);
            r.count = blocks ? int((start + uint32_t(blocks) - 1) / uint32_t(chunk) - unit) + 1 : 0;
            r.part = int(g / uint32_t(chunk)) + r.seq;
            return r;
        }
        before = uint32_t(__builtin_amdgcn_readlane(int(upto), 63));
    }
    return r;
}
// The shares of a unit, one after the other, or its one piece.
struct Shares {
    uint32_t at, end;
    int chunk;  // 0: a piece
};
__device__ __forceinline__ Shares first_share(const PagedArgs &a, int *err) {
    const Spread sp = spread(a, blockIdx.z == 0 ? err : nullptr);
    if (sp.chunk < kShare) return Shares{0, 1, 0};
    const unsigned long long at = blockIdx.z * (unsigned long long)sp.chunk, total = sp.total;
    return Shares{uint32_t(min(at, total)), uint32_t(min(at + sp.chunk, total)), sp.chunk};
}
__device__ __forceinline__ bool next_share(const PagedArgs &a, Shares &w, Share &r, int *err) {
    if (w.at >= w.end) return false;
    if (w.chunk) {
        r = share_at(a, w.chunk, w.at, w.end, -1);
        w.at += uint32_t(r.end - r.first);
        return true;
    }
    w.at = w.end;
    r = this_piece(a, nullptr);
    return r.count > 0;
}
// For the joins: the parts of a sequence.
__device__ __forceinline__ Piece split_piece(const PagedArgs &a, int want, bool, int *) {
    Share r{};
    const int chunk = a.shares ? spread(a, nullptr).chunk : 0;
    if (chunk >= kShare) r = share_at(a, chunk, 0, 0, want);
    else r = piece_share(a, want, false, nullptr);
    Piece p{};
    p.s = r.s;
    p.seq = want;
    p.first = r.part;
    p.count = r.count;
    return p;
}

// What a row (of token i) sees: positions up to `hi` that are above `lo` or among the first; with a tree, of the drafted
// tokens those whose bits are set (none for a row of padding).
struct RowView {
    int i, hi, lo;
};
__device__ __forceinline__ const uint32_t *row_bits(const PagedArgs &a, const Seq &s, int i) {
    return a.tree + size_t(s.t0 + i) * a.tree_words;
}
__device__ __forceinline__ RowView row_view(const PagedArgs &a, const Seq &s, int i) {
    const int cached = s.len - s.n, row = cached + i;
    RowView v{i, row, row - a.window};
    if (a.tree) {
        const uint32_t *bits = row_bits(a, s, i);
        int set = 0;
#pragma unroll 4
        for (int w = 0; 32 * w < s.n; ++w) set += __popc(bits[w] & (s.n - 32 * w < 32 ? (1u << (s.n - 32 * w)) - 1 : ~0u));
        v.hi = row < 0 ? -1 : cached - 1;
        v.lo = cached - 1 + max(set, 1) - a.window;
    }
    if (!a.window) v.lo = -1;
    return v;
}
// Whether the row sees position p of the sequence, drafted tokens of a tree aside.
__device__ __forceinline__ bool row_sees(const PagedArgs &a, const RowView &v, int p) {
    return (p <= v.hi) & ((p > v.lo) | (p < a.sinks));
}
// Bit i: whether the row sees position p + i (i < 32) as a drafted token of a tree.
__device__ __forceinline__ uint32_t row_drafts(const PagedArgs &a, const Seq &s, const RowView &v, int p) {
    const int cached = s.len - s.n, first = p - cached;
    if (!a.tree || first + 31 < 0) return 0;
    const uint32_t *bits = row_bits(a, s, v.i);
    const int words = (s.n + 31) >> 5, w = first >> 5;
    const uint32_t tail = s.n & 31 ? (1u << (s.n & 31)) - 1 : ~0u;
    uint32_t lo = 0, hi = 0;
    if (w >= 0 && w < words) lo = bits[w] & (w == words - 1 ? tail : ~0u);
    if (w + 1 < words) hi = bits[w + 1] & (w + 1 == words - 1 ? tail : ~0u);
    const uint32_t m = uint32_t(((uint64_t(hi) << 32) | lo) >> (first & 31));
    return cached + v.i < 0 ? 0 : m;
}
// Whether every one of rows i0..i1 sees all of positions p..p + count - 1.
__device__ __forceinline__ bool all_visible(const PagedArgs &a, const Seq &s, int i0, int i1, int p, int count) {
    const int cached = s.len - s.n, end = a.tree ? cached : cached + i0 + 1;
    const int last = a.tree ? s.len - 1 : cached + i1;  // (a drafted token's position is at most the last one)
    return cached + i0 >= 0 && p + count <= end && (!a.window || p > last - a.window || p + count <= a.sinks);
}

// The blocks that some of rows row..row_end - 1 sees, and of these (numbered as there) the share's: first, end.  Shares are
// cut by the sequence's blocks z.  Where rows see more first blocks than z has (their window has left them behind),
// z has no gap and its numbers are the blocks'.
__device__ __forceinline__ int2 tile_blocks(const PagedArgs &a, const Share &sh, const Seen &z, int row, int row_end, Seen &t) {
    const Seq &s = sh.s;
    const int p_first = s.len - s.n + row / a.group;
    const int p_last = a.tree ? s.len - 1 : s.len - s.n + (row_end - 1) / a.group;
    t = z;
    if (p_last < 0 || z.count == 0) return make_int2(0, 0);
    if (a.window && !a.tree) {  // (rows of a tree stand in no order)
        t.from = max(0, p_first - a.window + 1);
        t.first = t.from / kPos;
        t.sink = min((min(a.sinks, t.from) + kPos - 1) / kPos, t.first);
    }
    const int cut = sh.first, first = t.first - z.first + z.sink, skip = first - t.sink;
    const int end = z.sink + p_last / kPos + 1 - z.first;
    const int cut_end = min(end, sh.end);
    return make_int2(cut < t.sink ? cut : max(cut, first) - skip, max(min(cut_end, t.sink), cut_end - skip));
}

// The sequence's row of the page table, read through the scalar cache: a vector load's result could only be waited for with
// all of the keys and values in flight before it.
typedef const __attribute__((address_space(4))) int32_t table_word;
struct Table {
    table_word *row;
    int n_pages, shift, last;  // last: of the sequence's positions
    // The entry of position p's page (any p: that of the last position behind it).
    __device__ __forceinline__ int32_t entry(int p) const { return row[min(p, last) >> shift]; }
};
__device__ __forceinline__ Table sequence_table(const PagedArgs &a, const Share &sh) {
    return Table{(table_word *)(a.table + size_t(sh.seq) * a.max_pages), a.pages.n_pages, a.pages.shift, max(sh.s.len - 1, 0)};
}
// Whether some token sees one of the 16 positions from p on, which lie in one page.
__device__ __forceinline__ bool half_seen(const PagedArgs &a, const Seq &s, const Seen &all, int p) {
    return (p < s.len) & ((p < a.sinks) | (p + 16 > all.from));
}

// x as TERMS bf16 operands, each rounding what the ones before leave.
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8 (&t)[TERMS]) {
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16(rest[2 * e], rest[2 * e + 1]);
            if (k + 1 < TERMS) {
                rest[2 * e] -= low_half(w[e]);
                rest[2 * e + 1] -= high_half(w[e]);
            }
        }
        t[k] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}
// 8 or 16 bytes, read once or again.
template <typename T, typename ONCE>
__device__ __forceinline__ T read(const uint8_t *p, ONCE) {
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) / 4)));
    const words *w = reinterpret_cast<const words *>(p);
    return __builtin_bit_cast(T, ONCE::value ? __builtin_nontemporal_load(w) : *w);
}
// Eight elements of a bf16 query, with the scale's sign.
__device__ __forceinline__ bf16x8 load_query(const PagedArgs &a, size_t at) {
    uint4 w = dev::load16(reinterpret_cast<const uint8_t *>(static_cast<const uint16_t *>(a.q) + at));
    const uint32_t flip = a.negate ? 0x80008000u : 0u;
    w.x ^= flip, w.y ^= flip, w.z ^= flip, w.w ^= flip;
    return __builtin_bit_cast(bf16x8, w);
}
// Where a pair of bf16 is not finite: all ones in its half.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// grid: (row tiles, key/value head, sequence), or with a target (key/value head, row tiles, units).
//
// out_r = sum_p 2^(unit (s_rp - m_r)) V_p / sum_p 2^(unit (s_rp - m_r)), m_r the running maximum, in one pass.  What bounds it
// are the cache's bytes, each of which is read once per tile of rows: 32 sequences of up to 16384 positions, 8 heads of 128, 4
// queries each (1.40 GB) 212 us, 6.6 TB/s; 128 sequences that see 1028 positions, 8 heads of 64 (272 MB) 48 us, 5.7 TB/s; of one
// token over 4096 positions (8.4 MB, 8.3 us and 3.8 for the join) the latencies of a launch, the table, the keys and the join.
// Rows come in tiles of 16, since the queries of a token's head are 8 as a rule: tiles of 32 would multiply as much again for
// nothing, and hold twice the outputs where registers hold the loads in flight.
//
// A value that is not finite would reach every row of the tile (0 times it is NaN): a wave that ends with outputs that are
// not finite goes over its positions once more, with such values as zeros and the outputs of the rows that see one NaN.
template <int NG, int NT, bool F32, bool SHARES>
__global__ __launch_bounds__(kAttBlock, NG * NT <= 2 ? 2 : 1) void paged_attend_kernel(PagedArgs a) {
    constexpr int d = NG * 64, QT = F32 ? 3 : 1, PT = F32 ? 3 : 2, ROWS = 16;
    constexpr int VE = NG % 2 ? 4 : 8, VG = d / (16 * VE);  // dims of a lane per group of products, groups
    __shared__ float4 out_sh[kAttWaves][ROWS][d / 4 + 1];
    __shared__ float max_sh[kAttWaves][ROWS], sum_sh[kAttWaves][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    const int tile = a.split.target ? blockIdx.y : blockIdx.x, h = a.split.target ? blockIdx.x : blockIdx.y;
    int *bad_batch = tile == 0 && h == 0 && threadIdx.x < 64 ? a.err : nullptr;
    Shares shares{};
    Share sh;
    if constexpr (SHARES) {
        shares = first_share(a, bad_batch);
        if (!next_share(a, shares, sh, bad_batch)) return;
    } else {
        sh = this_piece(a, bad_batch);
        if (sh.count == 0) return;
    }
    do {
        const Seq &s = sh.s;
        const int G = a.group, rows = s.n * G, row0 = tile * ROWS * NT;
        if (row0 >= rows) continue;
        const int i_first = row0 / G, i_last = min(s.n - 1, (row0 + ROWS * NT - 1) / G);
        const Seen all = seen(s, a.window, a.sinks);
        Seen z;
        const int2 range = tile_blocks(a, sh, all, row0, min(row0 + ROWS * NT, rows), z);
        const Table table = sequence_table(a, sh);
        const int page_mask = (1 << a.pages.shift) - 1;

        // A block's operands as they lie in the cache: keys as 16 positions of 8 dims, values as 8 positions of VE dims.  The next
        // block's are loaded as soon as the present ones have been used: the bytes in flight are what bounds a batch of single
        // tokens.  (Two blocks at a time: the same over long caches; 256 sequences of up to 500 positions, 8 heads of 64 36 us, 34
        // with one; a window of 256 35 and 29, since more waves have nothing to do in a sequence's last blocks.)
        uint4 kc[2][2 * NG];
        uint32_t vc[VG][8][VE / 2];
        // Half a block lies in one page.  `there`: bits of the halves (four each) of which some token sees a position, and whose
        // page is there; the others are read from the first page, and none of it is used.  The table's entries are fetched a
        // block ahead of the loads.
        uint32_t there = 0;
        bool missing = false;
        int32_t entry[2] = {};
        int page_at[2] = {};
        auto block_at = [&](int v) { return z.block(min(v, range.y - 1)); };
        auto fetch = [&](int v) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 2; ++e) entry[e] = table.entry(block_at(v) * kPos + 16 * e);
        };
        auto find = [&](int v) __attribute__((always_inline)) {
            there = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool needed = half_seen(a, s, all, block_at(v) * kPos + 16 * e);
                const bool ok = uint32_t(entry[e]) < uint32_t(table.n_pages);
                missing |= needed & !ok;
                page_at[e] = ok ? entry[e] : 0;
                there |= needed && ok ? 0xfu << (4 * e) : 0u;
            }
        };
        // 16 positions of a block lie in a page: a base for all lanes, and offsets that stay.
        const uint8_t *head_k = reinterpret_cast<const uint8_t *>(a.pages.k + ((size_t(h) << a.pages.shift) * d));
        const uint8_t *head_v = reinterpret_cast<const uint8_t *>(a.pages.v + ((size_t(h) << a.pages.shift) * d));
        const uint32_t page_k = uint32_t(a.pages.k_stride) * 2, page_v = uint32_t(a.pages.v_stride) * 2;  // bytes (below 2^32)
        // Bytes that no other block reads pass through the caches as a stream, others stay there (32 sequences of up to 16384
        // positions, one token each: 220 us, 246 through the caches; 1000 tokens over 2000 positions in fp32, 32 heads over 8 of
        // 128: 141 us, 193 as a stream).
        const bool alone = a.tiles == 1;
        auto once_or_again = [&](auto load) __attribute__((always_inline)) {
            if (alone) {  // (between fences, as the compiler would make one of the two)
                asm volatile("" ::: "memory");
                load(std::true_type());
                asm volatile("" ::: "memory");
            } else {
                load(std::false_type());
            }
        };
        const uint32_t k_lane = 2 * (n * d + 8 * c), v_lane = 2 * (4 * c * d + VE * n);
        auto load_k = [&](int v) __attribute__((always_inline)) {
            const int at = block_at(v) * kPos;
            auto load = [&](auto once) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint8_t *src = head_k + (uint64_t(uint32_t(page_at[e])) * page_k + uint32_t((at + 16 * e) & page_mask) * (2 * d));
#pragma unroll
                    for (int j = 0; j < 2 * NG; ++j) kc[e][j] = read<uint4>(src + k_lane + 64 * j, once);
                }
            };
            once_or_again(load);
        };
        auto load_v = [&](int v) __attribute__((always_inline)) {
            const int at = block_at(v) * kPos;
            auto load = [&](auto once) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = i >> 2;
                    const uint8_t *src = head_v + (uint64_t(uint32_t(page_at[e])) * page_v + uint32_t((at + 16 * e) & page_mask) * (2 * d));
#pragma unroll
                    for (int g = 0; g < VG; ++g) {
                        const auto w = read<std::conditional_t<VE == 8, uint4, uint2>>(src + v_lane + 2 * d * (i & 3) + 32 * VE * g, once);
                        vc[g][i][0] = w.x, vc[g][i][1] = w.y;
                        if constexpr (VE == 8) vc[g][i][2] = w.z, vc[g][i][3] = w.w;
                    }
                }
            };
            once_or_again(load);
        };

        // The tile's rows: their queries as operands (k = dims), what they see.  A row past the last repeats it and is not stored.
        auto row_of = [&](int t) { return min(row0 + 16 * t + n, rows - 1); };
        const float sign = a.negate ? -1.f : 1.f;
        bf16x8 bq[NT][2 * NG][QT];
        RowView view[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = row_of(t), i = row / G;
            const size_t at = size_t(s.t0 + i) * a.q_stride + size_t(h * G + row - i * G) * d + 8 * c;
            view[t] = row_view(a, s, i);
#pragma unroll
            for (int j = 0; j < 2 * NG; ++j) {
                if constexpr (F32) {
                    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(a.q) + at + 32 * j);
                    const float4 u = p[0], w = p[1];
                    const float x[8] = {u.x * sign, u.y * sign, u.z * sign, u.w * sign, w.x * sign, w.y * sign, w.z * sign, w.w * sign};
                    split_terms<QT>(x, bq[t][j]);
                } else {
                    bq[t][j][0] = load_query(a, at + 32 * j);
                }
            }
        }
        floatx4 acc[NT][4 * NG];
        float mx[NT], sum[NT];
        auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                mx[t] = -INFINITY;
                sum[t] = 0.f;
#pragma unroll
                for (int i = 0; i < 4 * NG; ++i) acc[t][i] = floatx4{0.f, 0.f, 0.f, 0.f};
            }
            if (range.x + wave < range.y) {
                fetch(range.x + wave);
                find(range.x + wave);
                load_k(range.x + wave);
                load_v(range.x + wave);
                fetch(range.x + wave + kAttWaves);
            }
#pragma unroll 1
            for (int v = range.x + wave; v < range.y; v += kAttWaves) {
                const int next = v + kAttWaves, at = block_at(v) * kPos;
                const uint32_t held = there;
                const bool full = held == 0xff && all_visible(a, s, i_first, i_last, at, kPos);
                // ---- scores
                float p[NT][8];
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = QT - 1; k >= 0; --k)
#pragma unroll
                            for (int j = 0; j < 2 * NG; ++j) y = mfma(__builtin_bit_cast(bf16x8, kc[e][j]), bq[t][j][k], y);
#pragma unroll
                        for (int r = 0; r < 4; ++r) p[t][4 * e + r] = y[r];
                    }
                __builtin_amdgcn_sched_barrier(0);
                if (next < range.y) {
                    find(next);
                    load_k(next);
                    fetch(next + kAttWaves);
                }
                __builtin_amdgcn_sched_barrier(0);
                // ---- softmax
                uint32_t sees[NT];
                bf16x8 bp[NT][PT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    sees[t] = 0xff;
                    if (!full) {
                        const uint32_t drafts = row_drafts(a, s, view[t], at) >> (4 * c);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int i = 16 * (k >> 2) + (k & 3);
                            const bool see = (row_sees(a, view[t], at + 4 * c + i) | (drafts >> i & 1)) & (held >> k & 1);
                            p[t][k] = see ? p[t][k] : -INFINITY;
                            if constexpr (decltype(careful)::value) sees[t] &= ~(uint32_t(!see) << k);
                        }
                    }
                    float top = p[t][0];
#pragma unroll
                    for (int k = 1; k < 8; ++k) top = fmaxf(top, p[t][k]);
                    const float was = mx[t], now = fmaxf(was, max_over_c(top)), to = now == -INFINITY ? 0.f : now;
                    if (__any(now > was)) {
                        const float f = __builtin_amdgcn_exp2f((was - to) * a.unit);
                        mx[t] = now;
                        sum[t] *= f;
#pragma unroll
                        for (int i = 0; i < 4 * NG; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[t][i][r] *= f;
                    }
                    // (differences first: right at any size of the scores)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        p[t][k] = __builtin_amdgcn_exp2f((p[t][k] - to) * a.unit);
                        sum[t] += p[t][k];
                    }
                    split_terms<PT>(p[t], bp[t]);
                }
                // ---- values
                if (!full) {
                    // Positions that no token sees may hold anything: zeros.
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int pos = at + 16 * (i >> 2) + 4 * c + (i & 3);
                        const bool keep = (held >> i & 1) & (pos < s.len) & ((pos >= all.from) | (pos < a.sinks));
#pragma unroll
                        for (int g = 0; g < VG; ++g)
#pragma unroll
                            for (int w = 0; w < VE / 2; ++w) vc[g][i][w] = keep ? vc[g][i][w] : 0;
                    }
                }
                bf16x8 seen_by[NT];
                if constexpr (decltype(careful)::value) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = (sees[t] >> (2 * e) & 1) * 0x3f80u | (sees[t] >> (2 * e + 1) & 1) * 0x3f800000u;
                        seen_by[t] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
                    }
                }
#pragma unroll
                for (int g = 0; g < VG; ++g)
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = __builtin_amdgcn_perm(vc[g][2 * k + 1][e / 2], vc[g][2 * k][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
                        const int i = g * VE + e;
                        if constexpr (decltype(careful)::value) {
                            uint32_t f[4];
                            bool any = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                f[k] = not_finite(w[k]);
                                w[k] &= ~f[k];
                                any |= f[k] != 0;
                                f[k] &= 0x3f803f80u;
                            }
                            if (__any(any))
#pragma unroll
                                for (int t = 0; t < NT; ++t) {
                                    const floatx4 met = mfma(__builtin_bit_cast(bf16x8, make_uint4(f[0], f[1], f[2], f[3])), seen_by[t],
                                                             floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                                    for (int r = 0; r < 4; ++r)
                                        if (met[r] > 0.f) acc[t][i][r] = NAN;
                                }
                        }
                        const bf16x8 va = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int k = PT - 1; k >= 0; --k) acc[t][i] = mfma(va, bp[t][k], acc[t][i]);
                    }
                __builtin_amdgcn_sched_barrier(0);
                if (next < range.y) load_v(next);
            }
        };
        pass(std::false_type());
        bool off = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4 * NG; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) off |= !(fabsf(acc[t][i][r]) < INFINITY);
        if (__builtin_expect(__any(off), 0)) pass(std::true_type());
        if (missing && lane == 0) atomicOr(a.err, kErrRange);

        // Join the waves, one tile of rows at a time.
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float l = sum_over_c(sum[t]);
            if (t) __syncthreads();
            if (c == 0) {
                max_sh[wave][n] = mx[t];
                sum_sh[wave][n] = l;
            }
            // (row m = 4 c + r of product e of group g is dim 16 VE g + VE m + e)
#pragma unroll
            for (int g = 0; g < VG; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < VE; e += 4) {
                        const int i = g * VE + e;
                        out_sh[wave][n][(16 * VE * g + VE * (4 * c + r) + e) / 4] =
                            make_float4(acc[t][i][r], acc[t][i + 1][r], acc[t][i + 2][r], acc[t][i + 3][r]);
                    }
            __syncthreads();
#pragma unroll 1
            for (int idx = threadIdx.x; idx < ROWS * (d / 4); idx += kAttBlock) {
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
                    const float f = max_sh[w][r] == -INFINITY && sum_sh[w][r] == 0.f ? 0.f : __builtin_amdgcn_exp2f((max_sh[w][r] - M) * a.unit);
                    const float4 u = out_sh[w][r][i4];
                    S = fmaf(f, sum_sh[w][r], S);
                    v.x = fmaf(f, u.x, v.x);
                    v.y = fmaf(f, u.y, v.y);
                    v.z = fmaf(f, u.z, v.z);
                    v.w = fmaf(f, u.w, v.w);
                }
                if (sh.count > 1) {
                    float *o = a.part + ((size_t(sh.part) * a.n_kv + h) * a.tiles * (ROWS * NT) + row) * (d + 4);
                    *reinterpret_cast<float4 *>(o + 4 * i4) = v;
                    if (i4 == 0) *reinterpret_cast<float4 *>(o + d) = make_float4(M, S, a.unit, 0.f);
                    continue;
                }
                const float inv = S == 0.f ? 0.f : 1.f / S;  // (a row that sees nothing: 0)
                v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
                store4<F32>(a.out, size_t(s.t0 + row / G) * a.out_stride + size_t(h * G + row % G) * d + 4 * i4, v);
            }
        }
        if constexpr (SHARES) __syncthreads();  // (the next share's waves join through the same LDS)
    } while (SHARES && next_share(a, shares, sh, bad_batch));
}

// ---- many rows (prompts, wide trees), bf16 tensors ---------------------------------------------------------------
//
// Where a block of positions meets hundreds of rows the arithmetic counts: a wave takes 32 rows, the 32x32x16 product does
// twice the work per operand read, and the waves of a block share 64 positions' keys and values through LDS.  They lie there
// as in the cache, a row of dims per position, with the pieces of 16 bytes of a row permuted by its number, so that what is
// read together lies in different banks; the values are read by the transposing LDS load, which hands a lane four positions
// of its dim.  The next positions are loaded into registers before the present ones are used and written behind them into
// the other of two buffers, where positions that no token sees become zeros.
//
// Probabilities are one bf16 term here (2^-8), and their sum is that of the rounded ones, so that a row's weights add up to
// one: a second term costs half as many matrix products again (2048 tokens over 8192 positions 326 us, 260 with one; six
// prompts over a window of 1000 84 and 69; 60 drafted tokens 37 and 34), for an error of 1.7e-3 beside 2.3e-3, the output's
// rounding included.
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 64;  // positions per step
// A maximum is followed once a score is past it by so much (log2 units): probabilities of up to 2^8 lose nothing.  Sums of 2^26
// of them with values of up to 2^100 would pass fp32, though: from kLarge on a block goes over its positions once more and
// follows every maximum (sums below 2^126), and what stays below it in the parts of a sequence (512 at most) adds up to less.
constexpr float kSlack = 8.f, kLarge = 0x1p112f;
// Scores from here on (log2 units) are far: a row's offset, a rounded product, is off by 2^-12 at 2^12.  A step that has
// one takes its exponentials of differences.
constexpr float kFar = 0x1p12f;

__device__ __forceinline__ floatx16 mfma32(bf16x8 a, bf16x8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Where piece `i` (16 bytes) of row `row` lies in the row.  Reads take 8 rows' same piece (keys), or four pieces of 8 rows
// (values, 4 neighbouring rows per 16 lanes): over 256 bytes of banks each meets a bank as rarely as it can.
template <int NG>
__device__ __forceinline__ int swizzle(int row) {
    return NG % 2 ? ((row >> 1 & 1) << 2) | (row >> 2 & 3) : ((row & 3) << 2) | (row >> 2 & 3);
}
// N products with an operand from LDS each, which is read AHEAD products in front of its use.  (Left to itself the compiler
// reads an operand, waits and multiplies: an LDS latency for each product.)
template <int AHEAD, typename READ>
__device__ __forceinline__ void read_first(uint4 (&w)[AHEAD], READ read) {
#pragma unroll
    for (int m = 0; m < AHEAD; ++m) w[m] = read(m);
}
template <int N, int AHEAD, typename READ, typename USE>
__device__ __forceinline__ void products(uint4 (&w)[AHEAD], READ read, USE use) {  // w: as of read_first
#pragma unroll
    for (int m = 0; m < N; ++m) {
        __builtin_amdgcn_sched_barrier(0);
        use(m, w[m % AHEAD]);
        if (m + AHEAD < N) w[m % AHEAD] = read(m + AHEAD);
    }
}
// A number that the compiler takes as it is: it would otherwise keep dozens of sums with it in registers, not the few numbers.
__device__ __forceinline__ int held_value(int v) {
    asm("" : "+v"(v));
    return v;
}
__device__ __forceinline__ int held_scalar(int v) {
    asm("" : "+s"(v));
    return v;
}
typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef __attribute__((address_space(3))) dev::u32x4 lds_u32x4;
__device__ __forceinline__ uint2 read_turned(const lds_byte *p) {
    typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)p));
}
__device__ __forceinline__ float other_half32(float v) {  // what f(own, lane ^ 32) takes
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return (threadIdx.x & 32) ? __uint_as_float(r[0]) : __uint_as_float(r[1]);
}
// Whether some of rows i0..i1 sees some of the block of positions at p.
__device__ __forceinline__ bool any_visible(const PagedArgs &a, const Seq &s, int i0, int i1, int p) {
    const int cached = s.len - s.n;
    if (a.tree) return p < s.len;
    return p <= cached + i1 && (!a.window || p + kPos - 1 > cached + i0 - a.window || p < a.sinks);
}

// grid: (row tiles, key/value head, sequence), or with a target (key/value head, row tiles, units); 32 WAVES rows per block.
//
// Eight waves are two to a SIMD and go in two groups half a step apart, a barrier between: while the one forms its products
// (the values of its last positions, the scores of the next), the other takes its exponentials.  Four waves of a block are
// one to a SIMD; another block, which runs in no step with it, fills the gaps; two others with heads of 64, whose registers
// leave room (six prompts over a window of 1000, 16 heads: 70 us, 80 with one other; six of 700 tokens, 32 heads: 32 and 39;
// 4096 tokens of one: 125 and 122).
//
// What bounds it: per 64 positions a wave of heads of 128 has 32 products of 33 cycles and 1000 cycles of lane arithmetic (an
// exponential per score takes 10, its difference, maximum, rounding and sum as many again), and two waves to a SIMD overlap
// them in part only.  2048 tokens behind 6144, 32 heads over 4 of 128 (241 GFLOP): 259 us, 0.93 PFLOP/s; a matrix product of
// 16384 rows and columns reaches 1.6 here.  Its 256 blocks, one to a unit, have 97 to 128 steps each, and the longest one's
// are its time (2048 tokens by themselves, 1 to 32 steps: 74 us, 0.46 PFLOP/s).  Six prompts of up to 1789 tokens over a window of 1000, 16 heads over 4 of 64 (33.5
// GFLOP): 69 us, the lane arithmetic of half as many products.  (Rows of 64 a wave, whose operands would serve twice, do not
// fit the registers: 606 us; one wave to a SIMD that has its own exponentials beside its products: 370.)
template <int NG, int WAVES>
__global__ __launch_bounds__(64 * WAVES, NG == 1 && WAVES == 4 ? 3 : NG <= 2 ? 2 : 1) void paged_prompt_kernel(PagedArgs a) {
    constexpr int d = NG * 64, THREADS = 64 * WAVES, ROWS = 32 * WAVES, PIECES = d / 8, ROW = 2 * d;
    constexpr int LOADS = kTile * PIECES / THREADS, KS = d / 16, TD = d / 32;
    constexpr int HALF = 16 * PIECES / 64;   // loads of a wave that make 16 positions
    constexpr bool TWO = WAVES == 8;
    constexpr int AHEAD = 4;                 // products whose operands are in flight
    constexpr int VBUF = TWO ? 3 : 2;        // (values are read a step after the keys)
    __shared__ uint4 k_sh[2][kTile * PIECES], v_sh[VBUF][kTile * PIECES];
    __shared__ alignas(16) uint32_t there_sh[VBUF][4];  // bits of the halves of the two blocks that are there
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, c = lane >> 5;
    // (the last rows see the most positions: their blocks start first)
    const int tile = a.tiles - 1 - int(a.split.target ? blockIdx.y : blockIdx.x), h = a.split.target ? blockIdx.x : blockIdx.y;
    const Share sh = this_piece(a, tile == a.tiles - 1 && h == 0 && tid < 64 ? a.err : nullptr);
    if (sh.count == 0) return;
    const Seq &s = sh.s;
    const int G = a.group, rows = s.n * G, row0 = tile * ROWS;
    if (row0 >= rows) return;
    const Seen all = seen(s, a.window, a.sinks);
    Seen z;
    const int2 range = tile_blocks(a, sh, all, row0, min(row0 + ROWS, rows), z);
    const int steps = (range.y - range.x + 1) / 2;
    const Table table = sequence_table(a, sh);
    const int page_mask = (1 << a.pages.shift) - 1;

    const uint8_t *head_k = reinterpret_cast<const uint8_t *>(a.pages.k + ((size_t(h) << a.pages.shift) * d));
    const uint8_t *head_v = reinterpret_cast<const uint8_t *>(a.pages.v + ((size_t(h) << a.pages.shift) * d));
    const uint32_t page_k = uint32_t(a.pages.k_stride) * 2, page_v = uint32_t(a.pages.v_stride) * 2;  // bytes (below 2^32)

    // Steps whose 64 positions lie together and are all seen by some token, none of them past the last: most of them, and
    // those that need no look at where their positions are (`plain`: first, end; positions there are p_plain + 64 i).
    const int p_plain = (range.x - z.sink + z.first) * kPos;
    const int2 plain = [&] {
        const int gap = max(z.sink - range.x, 0);                                    // blocks in front of the window's
        const int unseen = a.window ? max(all.from - p_plain, 0) : 0;                // positions in front of the first seen
        return make_int2(max((gap + 1) / 2, (unseen + kTile - 1) / kTile), min((s.len - p_plain) / kTile, (range.y - range.x) / 2));
    }();
    auto half_at = [&](int i, int u) {  // where half u of step i's two blocks is
        return z.block(min(range.x + 2 * i + (u >> 1), range.y - 1)) * kPos + 16 * (u & 1);
    };

    // ---- staging: load l of a wave is 64 pieces of one half of a block, which lies in one page, in one piece
    uint4 kr[LOADS], vr[LOADS];
    int32_t entry[LOADS];     // the table's entries of the positions after those loaded
    bool there[LOADS];        // (careful) whether the loaded positions' half of a block is needed, and there
    uint32_t hold = 0;        // bit l: this thread's row of the loaded positions is seen by some token, and there
    bool missing = false;
    auto half_of = [&](int l) { return (l * WAVES + wave) / HALF; };
    auto piece_in = [&](int l) { return (l * THREADS + tid) % (16 * PIECES); };  // this thread's, of the half
    // Where in a buffer (bytes) the thread's pieces go, and its operands lie: keys of position n, values of dims of 16 lanes
    int k_off[KS], v_off[TD][2], store_at[LOADS];
    {
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
            const int row = piece_in(l) / PIECES;
            store_at[l] = held_value(16 * (16 * PIECES * half_of(l) + row * PIECES + ((piece_in(l) % PIECES) ^ swizzle<NG>(row))));
        }
        const int v_row = 4 * c + (lane & 15) / 4, v_piece = 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
#pragma unroll
        for (int j = 0; j < KS; ++j) k_off[j] = held_value(n * ROW + 16 * ((2 * j + c) ^ swizzle<NG>(n)));
#pragma unroll
        for (int t = 0; t < TD; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                v_off[t][e] = held_value((v_row + 8 * e) * ROW + 16 * ((4 * t + v_piece) ^ swizzle<NG>(v_row + 8 * e)) + 8 * (lane & 1));
    }

    auto fetch = [&](int i) __attribute__((always_inline)) {
        const bool easy = i >= plain.x && i < plain.y;
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
            entry[l] = table.row[(easy ? p_plain + kTile * i + 16 * half_of(l) : min(half_at(i, half_of(l)), table.last)) >> table.shift];
    };
    // easy: positions i are plain
    auto load = [&](int i, int l, bool easy, auto careful) __attribute__((always_inline)) {
        int p0 = p_plain + kTile * i + 16 * half_of(l);
        const bool ok = uint32_t(entry[l]) < uint32_t(table.n_pages);
        bool needed = true, keep = true;
        if (!easy) {
            p0 = half_at(i, half_of(l));
            needed = half_seen(a, s, all, p0);
            const int p = p0 + piece_in(l) / PIECES;
            keep = (p < s.len) & ((p >= all.from) | (p < a.sinks));
        }
        missing |= needed & !ok;
        if constexpr (decltype(careful)::value) {
            there[l] = needed & ok;
            keep &= ok;
        }
        hold = keep ? hold | 1u << l : hold & ~(1u << l);
        const uint64_t page = ok ? uint32_t(entry[l]) : 0u;
        const uint32_t at = uint32_t(p0 & page_mask) * ROW + 16u * uint32_t(piece_in(l));
        kr[l] = dev::load16(head_k + page * page_k + at);
        vr[l] = dev::load16(head_v + page * page_v + at);
    };
    auto store = [&](int i, int l, auto careful) __attribute__((always_inline)) {
        const int k_buf = held_scalar((i & 1) * int(sizeof k_sh[0])), v_buf = held_scalar(i % VBUF * int(sizeof v_sh[0]));
        const dev::u32x4 zero = {0, 0, 0, 0};
        *(lds_u32x4 *)((lds_byte *)k_sh[0] + k_buf + store_at[l]) = __builtin_bit_cast(dev::u32x4, kr[l]);
        *(lds_u32x4 *)((lds_byte *)v_sh[0] + v_buf + store_at[l]) = hold >> l & 1 ? __builtin_bit_cast(dev::u32x4, vr[l]) : zero;
        if constexpr (decltype(careful)::value)
            if ((l * WAVES + wave) % HALF == 0 && lane == 0) there_sh[i % VBUF][half_of(l)] = there[l] ? 1u << half_of(l) : 0u;
    };
    // The loaded positions (step i) go to LDS, those of the next are loaded, the table's entries of the one after fetched.
    auto stage = [&](int i, auto careful) __attribute__((always_inline)) {
        if (i >= steps) return;
#pragma unroll
        for (int l = 0; l < LOADS; ++l) store(i, l, careful);
        if (i + 1 >= steps) return;
#pragma unroll
        for (int l = 0; l < LOADS; ++l) load(i + 1, l, i + 1 >= plain.x && i + 1 < plain.y, careful);
        fetch(min(i + 2, steps - 1));
    };
    // The same where these steps are plain, a piece of it behind each of the first few products.
    auto stage_plain = [&](int i, int piece) __attribute__((always_inline)) {
        if (piece < LOADS) {
            hold = ~0u;
            store(i, piece, std::false_type());
        } else if (piece < 2 * LOADS) {
            load(i + 1, piece - LOADS, true, std::false_type());
        }
    };
    auto fetch_plain = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int l = 0; l < LOADS; ++l) entry[l] = table.row[uint32_t(p_plain + kTile * i + 16 * half_of(l)) >> table.shift];
    };

    // ---- the wave's rows; a row past the last repeats it and is not stored
    const int w_row0 = row0 + 32 * wave, row = min(w_row0 + n, rows - 1), i_row = row / G;
    const bool idle = w_row0 >= rows;
    const int i_first = min(w_row0, rows - 1) / G, i_last = min(w_row0 + 31, rows - 1) / G;
    bf16x8 bq[KS];
    {
        const size_t at = size_t(s.t0 + i_row) * a.q_stride + size_t(h * G + row - i_row * G) * d + 8 * c;
#pragma unroll
        for (int j = 0; j < KS; ++j) bq[j] = load_query(a, at + 16 * j);
    }
    const RowView view = row_view(a, s, i_row);

    floatx16 acc[TD], p[2];
    bf16x8 bp[4];
    uint32_t sees[2] = {0, 0};
    float mx, sum;
    // Steps that are plain and whose positions every row of the wave sees (first, end): they need no mask.
    const int2 whole = [&] {
        const int cached = s.len - s.n, end = a.tree ? cached : cached + i_first + 1, last = a.tree ? s.len - 1 : cached + i_last;
        int x = plain.x;
        if (a.window) x = max(x, max(0, last - a.window + 1 - p_plain + kTile - 1) / kTile);
        return make_int2(x, cached + i_first < 0 ? 0 : min(plain.y, (end - p_plain) / kTile));
    }();
    // Whether the wave has work at step i.
    auto live = [&](int i) {
        if (i >= whole.x && i < whole.y) return !idle;
        const int v = range.x + 2 * i;
        return !idle && (any_visible(a, s, i_first, i_last, z.block(v) * kPos) ||
                         (v + 1 < range.y && any_visible(a, s, i_first, i_last, z.block(v + 1) * kPos)));
    };
    // Scores: positions x rows, the two halves in turn, so that their sums do not wait for one another.
    auto keys_at = [&](int i) { return (const lds_byte *)k_sh[0] + held_scalar((i & 1) * int(sizeof k_sh[0])); };
    auto key = [&](const lds_byte *kb, int m) __attribute__((always_inline)) {
        return __builtin_bit_cast(uint4, *(const lds_u32x4 *)(kb + k_off[m >> 1] + (m & 1) * 32 * ROW));
    };
    auto score = [&](int m, uint4 w) __attribute__((always_inline)) {
        if (m < 2)
#pragma unroll
            for (int r = 0; r < 16; ++r) p[m][r] = 0.f;
        p[m & 1] = mfma32(__builtin_bit_cast(bf16x8, w), bq[m >> 1], p[m & 1]);
    };
    auto scores = [&](int i) __attribute__((always_inline)) {
        const lds_byte *kb = keys_at(i);
        uint4 w[AHEAD];
        read_first(w, [&](int m) { return key(kb, m); });
        products<2 * KS>(w, [&](int m) { return key(kb, m); }, score);
    };
    auto softmax = [&](int i, auto careful, auto masked) __attribute__((always_inline)) {
        sees[0] = sees[1] = 0xffff;
        uint32_t held = 0xf;
        if constexpr (decltype(careful)::value) {
            const uint4 halves = *reinterpret_cast<const uint4 *>(there_sh[i % VBUF]);
            held = __builtin_amdgcn_readfirstlane(halves.x | halves.y | halves.z | halves.w);
        }
        if (decltype(masked)::value && (i < whole.x || i >= whole.y || held != 0xf)) {
            const int v = range.x + 2 * i;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int at = z.block(min(v + u, range.y - 1)) * kPos;
                const uint32_t drafts = row_drafts(a, s, view, at) >> (4 * c);
                uint32_t m = 0;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = 8 * (r >> 2) + (r & 3);
                    const bool see = (row_sees(a, view, at + 4 * c + i) | (drafts >> i & 1)) &
                                     (held >> (2 * u + (r >> 3)) & 1) & (v + u < range.y);
                    p[u][r] = see ? p[u][r] : -INFINITY;
                    if constexpr (decltype(careful)::value) m |= uint32_t(see) << r;
                }
                if constexpr (decltype(careful)::value) sees[u] = m;
            }
        }
        float top = p[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, p[u][r]);
        top = fmaxf(top, other_half32(top));
        if (__any((top - mx) * a.unit > (decltype(careful)::value ? 0.f : kSlack))) {  // (the first score of a row is infinitely far past its maximum)
            const float now = fmaxf(mx, top), f = __builtin_amdgcn_exp2f(mx == now ? 0.f : (mx - now) * a.unit);
            mx = now;
            sum *= f;
#pragma unroll
            for (int t = 0; t < TD; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t][r] *= f;
        }
        const float to = mx == -INFINITY ? 0.f : mx;
        float off = to * a.unit;
        if (__any(!(fabsf(off) < kFar))) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) p[u][r] -= to;
            off = 0.f;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) p[u][r] = __builtin_amdgcn_exp2f(fmaf(p[u][r], a.unit, -off));
            uint32_t w[8];
            const bf16x2 one = {__bf16(1.f), __bf16(1.f)};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = pack_bf16(p[u][2 * e], p[u][2 * e + 1]);
                sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[e]), one, sum, false);
            }
            bp[2 * u] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
            bp[2 * u + 1] = __builtin_bit_cast(bf16x8, make_uint4(w[4], w[5], w[6], w[7]));
        }
    };
    // Outputs: dims x rows.
    auto values_at = [&](int i) { return (const lds_byte *)v_sh[0] + held_scalar(i % VBUF * int(sizeof v_sh[0])); };
    auto value = [&](const lds_byte *vb, int m) __attribute__((always_inline)) {
        const int q = m / TD, t = m % TD;
        const uint2 lo = read_turned(vb + v_off[t][0] + 16 * q * ROW), hi = read_turned(vb + v_off[t][1] + 16 * q * ROW);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    };
    auto output = [&](int m, uint4 w, auto careful) __attribute__((always_inline)) {
        const int q = m / TD, t = m % TD;
        if constexpr (decltype(careful)::value) {
            uint32_t x[4] = {w.x, w.y, w.z, w.w}, f[4], g[4];
            bool any = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[k] = not_finite(x[k]);
                x[k] &= ~f[k];
                any |= f[k] != 0;
                f[k] &= 0x3f803f80u;
                const uint32_t b = sees[q >> 1] >> (8 * (q & 1) + 2 * k);
                g[k] = (b & 1) * 0x3f80u | (b >> 1 & 1) * 0x3f800000u;
            }
            w = make_uint4(x[0], x[1], x[2], x[3]);
            if (__any(any)) {
                floatx16 met;
#pragma unroll
                for (int r = 0; r < 16; ++r) met[r] = 0.f;
                met = mfma32(__builtin_bit_cast(bf16x8, make_uint4(f[0], f[1], f[2], f[3])),
                             __builtin_bit_cast(bf16x8, make_uint4(g[0], g[1], g[2], g[3])), met);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (met[r] > 0.f) acc[t][r] = NAN;
            }
        }
        acc[t] = mfma32(__builtin_bit_cast(bf16x8, w), bp[q], acc[t]);
    };
    auto values = [&](int i, auto careful, auto beside) __attribute__((always_inline)) {  // beside(m): behind product m
        const lds_byte *vb = values_at(i);
        uint4 w[AHEAD];
        read_first(w, [&](int m) { return value(vb, m); });
        products<4 * TD>(w, [&](int m) { return value(vb, m); },
                         [&](int m, uint4 x) __attribute__((always_inline)) {
                             output(m, x, careful);
                             beside(m);
                         });
    };
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    auto pass = [&](auto careful) __attribute__((always_inline)) {
        mx = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int t = 0; t < TD; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
        if (steps > 0) {
            fetch(0);
#pragma unroll
            for (int l = 0; l < LOADS; ++l) load(0, l, false, careful);
            fetch(min(1, steps - 1));
            stage(0, careful);
        }
        lds_barrier();
        auto nothing = [](int) {};
        // Steps easy.x up to easy.y: plain ones, with plain ones behind them as far as staging reaches, seen whole by the
        // wave's rows.
        const int2 easy = decltype(careful)::value || idle ? make_int2(0, 0) : make_int2(whole.x + 1, min(whole.y, plain.y - 3));
        if constexpr (TWO) {
            // Step i of the first group: products in phase 2 i, exponentials in 2 i + 1; of the second one phase later.
            // Positions i + 1 are written beside step i's products, in phases 2 i and 2 i + 1: the last readers of the
            // buffers are through with phase 2 i - 1.
            const bool second = wave >= WAVES / 2;
            if (second) lds_barrier();
            bool was = false;
            auto step = [&](int i) __attribute__((always_inline)) {
                const bool now = i < steps && live(i);
                stage(i + 1, careful);
                fence();
                if (was) values(i + VBUF - 1, careful, nothing);
                if (now) scores(i);
                fence();
                lds_barrier();
                if (now) softmax(i, careful, std::true_type());
                fence();
                lds_barrier();
                was = now;
            };
            int i = 0;
#pragma unroll 1
            for (; i <= steps && i < easy.x; ++i) step(i);
            if constexpr (!decltype(careful)::value)
#pragma unroll 1
                for (; i < easy.y; ++i) {
                    const lds_byte *vb = values_at(i + VBUF - 1), *kb = keys_at(i);
                    auto operand = [&](int m) __attribute__((always_inline)) { return m < 4 * TD ? value(vb, m) : key(kb, m - 4 * TD); };
                    uint4 w[AHEAD];
                    read_first(w, operand);
                    products<4 * TD + 2 * KS>(w, operand, [&](int m, uint4 x) __attribute__((always_inline)) {
                        if (m < 4 * TD) output(m, x, careful);
                        else score(m - 4 * TD, x);
                        stage_plain(i + 1, m);
                    });
                    fence();
                    lds_barrier();
                    fence();
                    // (here, where no LDS read waits for the scalar cache)
                    fetch_plain(i + 3);
                    softmax(i, careful, std::false_type());
                    fence();
                    lds_barrier();
                }
#pragma unroll 1
            for (; i <= steps; ++i) step(i);
            if (!second) lds_barrier();
        } else {
            auto step = [&](int i) __attribute__((always_inline)) {
                if (live(i)) {
                    scores(i);
                    fence();
                    softmax(i, careful, std::true_type());
                    fence();
                    values(i, careful, nothing);
                }
                fence();
                stage(i + 1, careful);
                lds_barrier();
            };
            int i = 0;
#pragma unroll 1
            for (; i < steps && i < easy.x; ++i) step(i);
            if constexpr (!decltype(careful)::value) {
#pragma unroll 1
                for (; i < easy.y; ++i) {
                    scores(i);
                    fence();
                    fetch_plain(i + 2);
                    softmax(i, careful, std::false_type());
                    fence();
                    values(i, careful, [&](int m) __attribute__((always_inline)) { stage_plain(i + 1, m); });
                    fence();
                    lds_barrier();
                }
                if (i < steps) fetch(min(i + 2, steps - 1));
            }
#pragma unroll 1
            for (; i < steps; ++i) step(i);
        }
    };
    pass(std::false_type());
    bool off = false;
#pragma unroll
    for (int t = 0; t < TD; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) off |= !(fabsf(acc[t][r]) < kLarge);
    if (__builtin_expect(__syncthreads_or((off && !idle) || missing), 0)) pass(std::true_type());
    if (missing && lane == 0) atomicOr(a.err, kErrRange);
    const float l = sum + other_half32(sum);
    if (w_row0 + n >= rows) return;
    if (sh.count > 1) {
        float *o = a.part + ((size_t(sh.part) * a.n_kv + h) * a.tiles * ROWS + row) * (d + 4);
#pragma unroll
        for (int t = 0; t < TD; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<float4 *>(o + 32 * t + 2 * r + 4 * c) = make_float4(acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]);
        if (c == 0) *reinterpret_cast<float4 *>(o + d) = make_float4(mx, l, a.unit, 0.f);
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const size_t at = size_t(s.t0 + i_row) * a.out_stride + size_t(h * G + row - i_row * G) * d + 4 * c;
#pragma unroll
    for (int t = 0; t < TD; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            store4<false>(a.out, at + 32 * t + 2 * r, make_float4(acc[t][r] * inv, acc[t][r + 1] * inv, acc[t][r + 2] * inv, acc[t][r + 3] * inv));
}

constexpr int kLeastMany = 8;  // blocks of positions of a piece, at least, in the kernel for many rows
constexpr int most_tiles(int d, bool f32) { return d <= 128 && !(f32 && d > 64) ? 2 : 1; }  // what a wave's registers hold
// Blocks that are taken to fill the device (the reasons stand in paged_plan).
constexpr int few_fill(int d, int tiles) { return d / 64 * tiles > 2 ? 256 : kTarget; }
constexpr int many_fill(int d, bool one_each) { return one_each || d > 128 ? 256 : 512; }

// What a call launches: from its sizes alone, since lengths are on the device (max_kv bounds them).
struct PagedPlan {
    int prompt;             // waves of the kernel for many rows, or 0
    int tiles;              // otherwise: tiles of 16 rows per wave
    int tile_rows, blocks;  // rows per block, blocks of the largest sequence's rows
    int target, least, units;
    bool shares;            // enough positions, if sequences are long, for shares
    size_t workspace;
};
PagedPlan paged_plan(int n_seq, int n_kv, int group, int d, int max_q, int max_kv, bool f32) {
    const long long rows = (long long)max_q * group;
    PagedPlan p{};
    int fill;
    // More than 32 rows: the kernel for many, except where that for few has little to do, all of it at once (`few` blocks, a unit
    // of the device each), since its blocks start faster.  Heads of 128 over up to 1024 positions: 64 tokens of 4 sequences, 8
    // queries a head, 500 positions 16.5 us, 22.4 in the kernel for many; 16 of 4 over 900 17.1 and 19.5; 80 of 4 over 500
    // (320 blocks) 29 and 22.5; 40 of 4 over 900 26 and 21; 25 of 32 sequences, 8 heads, 300 positions 51 and 20.  Longer ones:
    // 5 of 4 over 4000 22 and 20; 16 of 8 over 8000, 8 heads 79 and 62.  Larger heads: 20 tokens of 2 sequences over 500, 4 queries
    // of 256 18 and 36; 60 of 2 over 2000 33 and 37; 100 of 2 over 2000 48 and 42; 20 of 32 over 2000 190 and 84.  Heads of 64: 10 tokens
    // of 8 sequences over 600 17.0 and 14.4.
    const long long few = (rows + (d > 128 ? 15 : 31)) / (d > 128 ? 16 : 32) * n_kv * n_seq;
    const bool little = d > 64 && few <= 256 && (d > 128 ? few * max_kv <= 1 << 18 : max_kv <= 1024 && few * max_kv <= 1 << 17);
    if (!f32 && rows > 32 && !little) {
        // Eight waves a block where their blocks fill the device once (2048 tokens, 32 heads over 4 of 128: 8192 positions 260 us,
        // 287 with four; 2048 positions 71 and 76; 1500 tokens of two sequences, 32 heads: 147 and 167; heads of 64, 8192
        // positions 164 and 178).  Where some of them run behind the others, smaller blocks even out (4096 tokens 221 us, 188 with
        // four; 3000 over 8192 427 and 393).
        const long long eight = (rows + 255) / 256 * n_kv * n_seq;
        p.prompt = d <= 128 && eight > 192 && eight <= 256 ? 8 : 4;
        p.tile_rows = 32 * p.prompt;
        p.least = kLeastMany;
        // Two blocks to a unit of the device; one where few rows are split into many pieces, whose outputs cost more than the
        // second gives (60 drafted tokens, 8 heads of 128, 8252 positions: 34 us, 40 with two; 16 tokens, 60000 positions: 58
        // and 63; sixteen sequences of 25, 4 heads: 70 us, 67 with two).
        const long long tiles = (rows + p.tile_rows - 1) / p.tile_rows * n_kv * n_seq;
        fill = many_fill(d, p.prompt == 8 || tiles <= 64);
    } else {
        // (a second tile halves the bytes of 17 rows and more, and needs as many registers again for its outputs)
        p.tiles = rows <= 16 ? 1 : most_tiles(d, f32);
        p.tile_rows = 16 * p.tiles;
        p.least = kAttWaves;
        // (where a wave's registers leave room for one block to a unit only: 4 tokens of 4 sequences over 4096 positions, 4 heads
        // of 128, 8 queries each 20 us, 28 with 512; 16 single tokens, 8 heads of 256: 91 and 97)
        fill = few_fill(d, p.tiles);
    }
    p.blocks = int((rows + p.tile_rows - 1) / p.tile_rows);
    const long long base = (long long)p.blocks * n_kv;  // blocks per sequence or piece
    const long long shares = ((max_kv - 1) / kPos + 1 + p.least - 1) / p.least;  // most that a sequence has
    if ((p.prompt ? base * n_seq * 2 <= fill : base * n_seq < fill) && max_kv > kWhole) {
        p.target = int(std::min(std::max(1ll, fill / base), shares * n_seq));
        p.units = p.target + n_seq - 1;  // (rounding up leaves less than one piece more per sequence)
        p.shares = !p.prompt && n_seq > 1 && (long long)n_seq * max_kv >= (long long)kShare * kPos * p.target;
        p.workspace = (size_t(p.units) * n_kv * p.blocks * p.tile_rows * (d + 4) * sizeof(float) + 255) & ~size_t(255);
    }
    return p;
}

}  // namespace

size_t paged_attention_call_bytes(int n_seq, int n_heads, int n_kv, int d, int max_q, int max_kv, bool f32) {
    return paged_plan(n_seq, n_kv, n_heads / n_kv, d, max_q, max_kv, f32).workspace;
}

// What a call asks for does not grow with its sizes: splits end where rows, heads and sequences fill the device, and the
// kernel for many rows begins at 33.  A caller sizes one workspace by the largest call, so this bounds what every call of at
// most these sizes asks for, kernel by kernel: units x base blocks (paged_plan) are target base + (n_seq - 1) base, of which the
// first is at most `fill` and what a piece's least positions leave, the second below what keeps a batch split.
size_t paged_attention_workspace_bytes(int n_seq, int n_heads, int n_kv, int d, int max_q, int max_kv) {
    if (max_kv <= kWhole) return 0;
    const long long rows = (long long)max_q * (n_heads / n_kv), blocks_kv = (max_kv - 1) / kPos + 1;
    auto bound = [&](int tile_rows, long long most_rows, int least, int fill, int rest) {
        const long long base = (std::min(rows, most_rows) + tile_rows - 1) / tile_rows * n_kv;
        const long long pieces = (blocks_kv + least - 1) / least * n_seq, most = fill;
        const long long units = std::min(most, std::min(most, pieces) * std::min(most, base)) + std::min<long long>(rest, (n_seq - 1) * base);
        return (size_t(units) * tile_rows * (d + 4) * sizeof(float) + 255) & ~size_t(255);
    };
    size_t n = 0;
    for (const bool f32 : {false, true}) {
        const int most = most_tiles(d, f32);
        const long long few = most == 1 ? rows : 16;
        n = std::max(n, bound(16, few, kAttWaves, few_fill(d, 1), few_fill(d, 1) - 1));
        if (rows > 16 && most > 1) n = std::max(n, bound(16 * most, rows, kAttWaves, few_fill(d, most), few_fill(d, most) - 1));
    }
    // (eight waves a block are never split)
    if (rows > 32) n = std::max(n, bound(32 * 4, rows, kLeastMany, many_fill(d, false), many_fill(d, false) / 2));
    return n;
}

hipError_t launch_paged_attention(const void *q, int dtype, long long q_stride, const paged::Pages &pages,
                                  const int32_t *table, int max_pages, const kv4::Batch &batch, int n_heads, int n_kv, int d,
                                  int window, int sinks, const uint64_t *tree, int tree_words, float scale, void *out,
                                  long long out_stride, void *workspace, int *err, hipStream_t s) {
    const bool f32 = dtype == MOE_F32;
    const PagedPlan p = paged_plan(batch.n_seq, n_kv, n_heads / n_kv, d, batch.max_q, batch.max_pos, f32);
    PagedArgs a;
    a.q = q;
    a.out = out;
    a.pages = pages;
    a.table = table;
    a.tree = reinterpret_cast<const uint32_t *>(tree);
    a.part = static_cast<float *>(workspace);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.max_pages = max_pages;
    a.tree_words = 2 * tree_words;
    a.n_kv = n_kv;
    a.group = n_heads / n_kv;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.tiles = p.blocks;
    // (never 0: -inf times it stays -inf)
    a.unit = std::max(std::fabs(scale) * 1.44269504088896341f, 0x1p-126f);
    a.negate = scale < 0.f;
    a.split.target = p.target;
    a.split.least = p.least;
    a.split.unit = p.prompt ? 2 : 1;
    a.shares = p.shares;
    a.batch = batch;
    a.err = err;
    const dim3 grid = p.target ? dim3(n_kv, p.blocks, p.units) : dim3(p.blocks, n_kv, batch.n_seq);
    if (p.prompt) {
#define PAGED_PROMPT(NG, W) \
    if (d == NG * 64 && p.prompt == W) paged_prompt_kernel<NG, W><<<grid, 64 * W, 0, s>>>(a);
        PAGED_PROMPT(1, 4) PAGED_PROMPT(1, 8) PAGED_PROMPT(2, 4) PAGED_PROMPT(2, 8) PAGED_PROMPT(3, 4) PAGED_PROMPT(4, 4)
#undef PAGED_PROMPT
    } else {
#define PAGED_CASE(NG, NT, F) \
    case (NG * 2 + F) * 8 + NT:                                               \
        if (p.shares) paged_attend_kernel<NG, NT, F, true><<<grid, kAttBlock, 0, s>>>(a); \
        else paged_attend_kernel<NG, NT, F, false><<<grid, kAttBlock, 0, s>>>(a);         \
        break;
    switch ((d / 64 * 2 + f32) * 8 + p.tiles) {
        PAGED_CASE(1, 1, false) PAGED_CASE(1, 2, false) PAGED_CASE(1, 1, true) PAGED_CASE(1, 2, true)
        PAGED_CASE(2, 1, false) PAGED_CASE(2, 2, false) PAGED_CASE(2, 1, true)
        PAGED_CASE(3, 1, false) PAGED_CASE(3, 1, true)
        PAGED_CASE(4, 1, false) PAGED_CASE(4, 1, true)
    default: return hipErrorInvalidValue;
    }
#undef PAGED_CASE
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.target) return e;
#define PAGED_JOIN(NG, F) \
    if (d == NG * 64 && f32 == F) launch_join<NG, F>(a, batch.max_q * a.group, batch.n_seq, p.tile_rows, s);
    PAGED_JOIN(1, false) PAGED_JOIN(1, true) PAGED_JOIN(2, false) PAGED_JOIN(2, true)
    PAGED_JOIN(3, false) PAGED_JOIN(3, true) PAGED_JOIN(4, false) PAGED_JOIN(4, true)
#undef PAGED_JOIN
    return hipGetLastError();
}

}  // namespace moe
