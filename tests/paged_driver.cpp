// Where a token of a paged cache is, and what a sentence's nodes can see: paged.hpp on the host.  Prints one line per query.
//   paged_driver offset N_PAGES PAGE_SHIFT MAX_PAGES PAGE_STRIDE TOKEN_STRIDE TABLE_STRIDE B T ENTRY...
//   paged_driver span PREFIX TREE LIMIT
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "../paper_1804_06609_amd/csrc/paged.hpp"

int main(int argc, char **argv)
{
    if (argc == 5 && !strcmp(argv[1], "span")) {
        const dba::Span s = dba::span_of(atoi(argv[2]), atoi(argv[3]), atoi(argv[4]));
        printf("%d %d\n", s.prefix, s.end);
        return 0;
    }
    if (argc < 10 || strcmp(argv[1], "offset")) return 2;
    std::vector<int32_t> table;
    for (int i = 10; i < argc; ++i) table.push_back(atoi(argv[i]));
    dba::Paged c;
    c.table = table.data();
    c.n_pages = atoi(argv[2]);
    c.page_shift = atoi(argv[3]);
    c.max_pages = atoi(argv[4]);
    c.page_stride = atoll(argv[5]);
    c.token_stride = atoll(argv[6]);
    c.head_stride = 0;
    c.table_stride = atoll(argv[7]);
    printf("%lld\n", (long long)dba::token_offset(c, atoi(argv[8]), atoll(argv[9])));
    return 0;
}
