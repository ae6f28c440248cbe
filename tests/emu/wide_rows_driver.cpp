// Edges of rows that take twelve and sixteen wavefronts, in workgroups that have more than one row: the same checks as the
// driver of small edges.
#define main small_main
#include "blocks_driver.cpp"
#undef main

int main(int argc, char **argv)
{
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "one") {        // two rows of one gate row, or of none: one workgroup
        edge(2, 8200, F, B, L, L, true, 2, false, true, 1);
        edge(2, 8200, H, H, R, L, true, 0, false, false, 0);
        edge(2, 10001, B, B, L, R, true, 2, true, false, 0);
        edge(2, 7001, F, F, L, L, true, 2, true, true, 0);
        edge(2, 5000, F, H, R, R, false, 0, false, false, 3);
    } else if (what == "many16") {     // more rows than workgroups
        edge(261, 8200, F, B, L, L, true, 0, false, true, 0);
    } else if (what == "many12") {
        edge(517, 4104, B, B, R, L, true, 2, false, true, 0);
    } else {
        return 2;
    }
    printf("%llu values as expected\n", (unsigned long long)checks);
    return 0;
}
