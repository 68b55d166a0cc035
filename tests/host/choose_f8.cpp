// Prints the kernels that a pointwise layer on FP8 blocks takes on 256 compute units: one "rows cin cout" per line; on codes and on 16-bit input.
#include "../../paper_2411_00288_amd/csrc/ss_f8_choice.h"
#include <cstdio>

int main()
{
    long long rows;
    int cin, cout;
    while (std::scanf("%lld %d %d", &rows, &cin, &cout) == 3) {
        const ss::F8Dims t = ss::f8_dims(cout, cin);
        const ss::F8Kernel k = ss::choose_f8_16(t, rows, 256);
        std::printf("%d %d %d %d\n", ss::choose_f8_codes(t, rows, 256), k, ss::f8_fits16(t, rows, k), ss::f8_rows_splits(t, rows, 256));
    }
    return 0;
}
