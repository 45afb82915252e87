// Prints the rows of groups of tokens read from stdin: token0 n first end heads a line.
#include <cstdio>

#include "rrq_append_rows.h"

int main()
{
    long long token0, first, end;
    int n, heads;
    while (std::scanf("%lld %d %lld %lld %d", &token0, &n, &first, &end, &heads) == 5) {
        const rrq_detail::GroupRows g = rrq_detail::group_rows(token0, n, first, end, heads);
        std::printf("%d %d %d\n", g.tokens, g.begin, g.end);
    }
    return 0;
}
