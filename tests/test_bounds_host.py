"""The rule by which the checked-access build lets an access through, on the host."""
import host_program


def test_an_access_is_inside_one_range_and_aligned_for_its_type(tmp_path):
    code, out = host_program.run(tmp_path, r"""
#include <cstdio>
#include "bounds_check.cuh"
int main()
{
    dass::BoundsTable t{};
    t.lo[0] = 0x1000; t.hi[0] = 0x1064;          // 100 bytes
    t.lo[1] = 0x2002; t.hi[1] = 0x2040;
    t.n = 2;
    const struct { unsigned long long a; unsigned n; bool ok; unsigned align; } cases[] = {                    // align 0: as wide as the access
        {0x1000, 16, true}, {0x1050, 16, true}, {0x1060, 16, false}, {0x1060, 4, true}, {0x1062, 2, true}, {0x1064, 1, false}, {0x0ff0, 16, false},
        {0x1008, 16, false}, {0x1004, 8, false}, {0x1002, 4, false}, {0x1001, 2, false}, {0x1001, 1, true},    // inside but not aligned
        {0x2002, 2, true}, {0x2002, 16, false}, {0x2004, 4, true}, {0x2000, 16, false}, {0x2030, 16, true},
        {0x1008, 24, true, 8}, {0x104c, 24, false, 8}, {0x1050, 24, false, 8}, {0x1008, 16, true, 8},              // a struct of 8-byte words
    };
    int wrong = 0;
    for (const auto &c : cases)
        if (dass::access_allowed(t, c.a, c.n, c.align ? c.align : c.n) != c.ok) { std::printf("%llx x %u\n", c.a, c.n); ++wrong; }
    return wrong;
}
""", flags=["-DDASS_BOUNDS_CHECK"])
    assert code == 0, out
