// What the kernels over a paged key/value cache share: the batch as they see it and the way from a position to its row.
//
// Pools are [pages][kv_heads][page][128] fp16, keys and values apart, so that a head's rows of a page are contiguous; a page holds
// 16 to 256 positions, a power of two.  Sequence b has seq_len[b] positions, in the pages that row b of the table names, and its
// last n = q_start[b + 1] - q_start[b] positions are the tokens of the call, rows q_start[b]... of its arrays.
#ifndef FQ_PAGED_H
#define FQ_PAGED_H

#include "fq_device.h"
#include "fq_internal.h"

constexpr int PD = 128; // head dimension

struct PagedSeqs {
    const int *q_start, *seq_len, *table;
    int seqs, tokens, max_len, table_stride, page_log2, pages;
};

inline PagedSeqs paged_seqs(const fq_paged_batch &b)
{
    int log2 = 4;
    while ((1 << log2) < b.page)
        ++log2;
    return PagedSeqs{b.q_start, b.seq_len, b.table, b.seqs, b.tokens, b.max_len, b.table_stride, log2, b.pages};
}

struct SeqRange {
    int first, n, len; // first token of the call's arrays, tokens, positions
};

// What the arrays say is cut to what the host has checked: whatever they hold, no access leaves the buffers.
__device__ __forceinline__ SeqRange seq_range(const PagedSeqs &p, int b)
{
    SeqRange s;
    s.first = min(max(p.q_start[b], 0), p.tokens);
    s.n = min(max(p.q_start[b + 1], s.first), p.tokens) - s.first;
    s.len = min(max(p.seq_len[b], 0), p.max_len);
    return s;
}

// Row of position t of sequence b in a pool's rows of one head of 128: (page * kv_heads + head) * page size + place in the page.
__device__ __forceinline__ size_t pool_row(const int *table, int table_stride, int page_log2, int pages, int kv_heads, int head, int b, int t)
{
    const int pg = table[(size_t)b * table_stride + min(t >> page_log2, table_stride - 1)];
    const int page = min(max(pg, 0), pages - 1);
    return ((((size_t)page * kv_heads + head) << page_log2) | (size_t)(t & ((1 << page_log2) - 1)));
}

// Sequence of token m: how many of q_start[1..seqs] are at most m.  One load a lane for 64 sequences, no chain of dependent ones.
// Every lane of the wavefront has the same m.
__device__ __forceinline__ int seq_of_token(const PagedSeqs &p, int m)
{
    const int lane = threadIdx.x & 63;
    int b = 0;
    for (int i = 0; i < p.seqs; i += 64) {
        const bool before = i + lane < p.seqs && p.q_start[1 + i + lane] <= m;
        b += (int)__popcll(__builtin_amdgcn_ballot_w64(before));
    }
    return min(b, p.seqs - 1);
}

#endif
