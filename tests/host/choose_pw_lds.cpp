// Prints, on 256 compute units, what a pointwise MXFP4 layer on 16-bit input takes (the kernel's id, the waves of a workgroup of 32 rows) and how many such workgroups LDS holds:
// one "rows cin cout" per line.
#include "../../paper_2411_00288_amd/csrc/ss_pw_choice.h"
#include <cstdio>

int main()
{
    long long rows;
    int cin, cout;
    while (std::scanf("%lld %d %d", &rows, &cin, &cout) == 3) {
        const ss::Mx4Dims t = ss::mx4_dims(cout, cin);
        std::printf("%d %d %d\n", ss::choose16(t, rows, 256), ss::rows_waves(t, rows, 256), (int)(ss::kPwLds / ss::rows_lds(t, 32)));
    }
    return 0;
}
