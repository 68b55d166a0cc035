// Prints whether a pointwise MXFP4 layer's output passes the caches by in the kernel with rows in LDS: one "rows cin cout residual" per line.
#include "../../paper_2411_00288_amd/csrc/ss_pw_choice.h"
#include <cstdio>

int main()
{
    long long rows;
    int cin, cout, residual;
    while (std::scanf("%lld %d %d %d", &rows, &cin, &cout, &residual) == 4)
        std::printf("%d\n", ss::rows_past_caches(ss::mx4_dims(cout, cin), rows, cout, residual != 0));
    return 0;
}
