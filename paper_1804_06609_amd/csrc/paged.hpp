// Where a token of a paged cache is.  Also compiled for the host, where its bounds are tested.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define DBA_HD __host__ __device__ __forceinline__
#else
#define DBA_HD inline
#endif

namespace dba {

struct Paged {
    const int32_t *table;              // of all sentences
    int64_t table_stride;
    int64_t page_stride, token_stride, head_stride;   // elements
    int n_pages, page_shift, max_pages;
};

// Offset in elements of head 0 of token t of sentence b; -1 if there is no such token or its page is not there.
DBA_HD int64_t token_offset(const Paged &c, int b, int64_t t)
{
    if (t < 0 || (t >> c.page_shift) >= c.max_pages) return -1;
    const int32_t page = c.table[(int64_t)b * c.table_stride + (t >> c.page_shift)];
    if ((uint32_t)page >= (uint32_t)c.n_pages) return -1;
    return (int64_t)page * c.page_stride + (t & (((int64_t)1 << c.page_shift) - 1)) * c.token_stride;
}

// What a sentence's nodes can see: tokens [0, prefix) all of them, [prefix, end) by the mask.
struct Span {
    int prefix, end;
};
DBA_HD Span span_of(int prefix, int tree, int limit)
{
    Span s;
    s.prefix = prefix < 0 ? 0 : prefix < limit ? prefix : limit;
    const int64_t end = (int64_t)(prefix < 0 ? 0 : prefix) + (tree < 0 ? 0 : tree);
    s.end = end < limit ? (int)end : limit;
    return s;
}

// The same of the nodes up to `last` of a chain of n, which is the last n of the tree's tokens.
DBA_HD Span span_of_chain(int prefix, int tree, int n, int last, int limit)
{
    Span s = span_of(prefix, tree, limit);
    const int64_t seen = (int64_t)(tree < 0 ? 0 : tree) - n + last + 1, end = s.prefix + (seen < 0 ? 0 : seen);
    if (end < s.end) s.end = (int)end;
    return s;
}

}  // namespace dba
