// What the operators' entry points and kernels work out about places in memory, on the host.  One query a line, one line an answer:
//   chain PREFIX TREE N LAST LIMIT
#include <stdio.h>
#include <string.h>

#include "../paper_1804_06609_amd/csrc/paged.hpp"

int main()
{
    char what[16];
    while (scanf("%15s", what) == 1) {
        if (strcmp(what, "chain")) return 2;
        int prefix, tree, n, last, limit;
        if (scanf("%d %d %d %d %d", &prefix, &tree, &n, &last, &limit) != 5) return 2;
        const dba::Span s = dba::span_of_chain(prefix, tree, n, last, limit);
        printf("%d %d\n", s.prefix, s.end);
    }
    return 0;
}
