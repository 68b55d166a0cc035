// Prints the waves of the few-row kernel of a pointwise MXFP4 layer on 16-bit input: one "rows cin cout" per line.
#include "../../paper_2411_00288_amd/csrc/ss_pw_choice.h"
#include <cstdio>

int main()
{
    long long rows;
    int cin, cout;
    while (std::scanf("%lld %d %d", &rows, &cin, &cout) == 3) std::printf("%d\n", ss::few16_waves(ss::mx4_dims(cout, cin), rows, cin));
    return 0;
}
