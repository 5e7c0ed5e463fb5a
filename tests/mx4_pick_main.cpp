// Prints the form and shape that the library picks for products read from
// standard input: n m groups d_in d_out by_expert gathered compute-units.
#include <cstdio>

#include "../paper_2603_04359_amd/csrc/mx4_pick.h"

int main() {
    int n, m, groups, d_in, d_out, by_expert, gathered, cus;
    while (std::scanf("%d %d %d %d %d %d %d %d", &n, &m, &groups, &d_in, &d_out, &by_expert, &gathered, &cus) == 8) {
        const catk::Mx4Sizes z{n, m, groups, d_in, d_out, by_expert != 0, gathered != 0};
        const catk::Mx4Pick p = catk::mx4_pick(z, cus);
        const char* form = p.form == catk::Mx4Form::split ? "split" : p.form == catk::Mx4Form::line ? "line" : "tile";
        std::printf("%s %d %d\n", form, p.shape, p.whole ? 1 : 0);
    }
    return 0;
}
