// What the operators' entry points and kernels work out about places in memory, on the host.  One query a line, one line an answer:
//   chain PREFIX TREE N LAST LIMIT
//   meet STEPS, then twice: AT LEN and COUNT STRIDE of three axes      (whether they have a byte in common, whether the first is nested)
#include <stdio.h>
#include <string.h>

#include "../paper_1804_06609_amd/csrc/paged.hpp"
#include "../paper_1804_06609_amd/csrc/places.hpp"

static bool places(dba::Places *p)
{
    long long at, len, count[3], stride[3];
    if (scanf("%lld %lld", &at, &len) != 2) return false;
    *p = dba::Places(reinterpret_cast<void *>(at), len);
    for (int i = 0; i < 3; ++i) {
        if (scanf("%lld %lld", &count[i], &stride[i]) != 2) return false;
        p->axis(count[i], stride[i]);
    }
    return true;
}

int main()
{
    char what[16];
    while (scanf("%15s", what) == 1) {
        if (!strcmp(what, "meet")) {
            int steps;
            dba::Places a, b;
            if (scanf("%d", &steps) != 1 || !places(&a) || !places(&b)) return 2;
            printf("%d %d\n", dba::meet(a, b, steps), a.nested());
            continue;
        }
        if (strcmp(what, "chain")) return 2;
        int prefix, tree, n, last, limit;
        if (scanf("%d %d %d %d %d", &prefix, &tree, &n, &last, &limit) != 5) return 2;
        const dba::Span s = dba::span_of_chain(prefix, tree, n, last, limit);
        printf("%d %d\n", s.prefix, s.end);
    }
    return 0;
}
