// paged.h -- the paged bf16 key/value cache: keys and values in pages of 2^m positions, [page][head][position][dim], and
// per sequence a row of page numbers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moe {
namespace paged {

struct Pages {
    uint16_t *k, *v;                // device bf16 [n_pages][n_kv][1 << shift][d], pages `k_stride`, `v_stride` elements apart
    long long k_stride, v_stride;
    int n_pages, shift;             // positions of a page: 1 << shift
};

struct TableArgs {
    const int32_t *kv_len, *n_new;  // [n_seq] positions held, tokens added (NULL: one each)
    const int32_t *free_pages, *free_first;
    int32_t *table, *kv_len_out, *q_start, *positions, *slots, *free_next;
    int n_seq, T, max_pages, shift, n_pages, n_free;
};

}  // namespace paged
}  // namespace moe
