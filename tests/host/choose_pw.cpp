// Prints the kernels that a pointwise MXFP4 layer takes on 256 compute units: one "rows cin cout" per line; on codes and on 16-bit input.
#include "../../paper_2411_00288_amd/csrc/ss_pw_choice.h"
#include <cstdio>

int main()
{
    long long rows;
    int cin, cout;
    while (std::scanf("%lld %d %d", &rows, &cin, &cout) == 3) {
        const ss::Mx4Dims t = ss::mx4_dims(cout, cin);
        const ss::PwKernel k = ss::choose16(t, rows, 256);
        std::printf("%d %d %d %d\n", ss::choose_codes(t, rows, 256), k, ss::fits16(t, rows, k), ss::rows_splits(t, rows, 256));
    }
    return 0;
}
