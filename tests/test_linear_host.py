"""When the epilogue of dass_linear may take whole 16-byte accesses, on the host: exactly where every address it would form
is aligned."""
import host_program

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "linear_common.cuh"
using namespace dass;
static const void *at(int64_t byte) { return reinterpret_cast<const void *>((uintptr_t)byte); }
static bool rows_aligned(const void *p, int64_t pitch, int64_t rows)
{
    for (int64_t r = 0; r < rows; ++r)
        if ((reinterpret_cast<uintptr_t>(p) + r * pitch * 2) % 16) return false;
    return true;
}
int main()
{
    int wrong = 0, wide = 0;
    for (int64_t N : {8, 96, 98, 100, 101, 102, 1028})
        for (int groups : {1, 2, 5})
            for (int64_t pad : {0, 1, 2, 3, 4, 12})
                for (int bias : {-1, 0, 4, 8})
                    for (int up : {-1, 0, 4, 8})
                        for (int res : {-1, 0, 8})
                            for (int y : {0, 4, 8}) {
                                LinearArgs a{};
                                a.T = 5; a.N = N; a.groups = groups; a.bf16 = true;
                                a.ldy = N + pad; a.ldr = N + pad;
                                a.Y = const_cast<void *>(at(4096 + y));
                                a.bias = bias < 0 ? nullptr : at(8192 + bias);
                                a.bias_up = up < 0 ? nullptr : at(16384 + up);
                                a.residual = res < 0 ? nullptr : at(32768 + res);
                                const bool all = rows_aligned(a.Y, a.ldy, a.T) && (!a.residual || rows_aligned(a.residual, a.ldr, a.T)) &&
                                                 (!a.bias || rows_aligned(a.bias, N, groups)) && (!a.bias_up || rows_aligned(a.bias_up, N, groups));
                                wide += all;
                                if (lin_wide_ok(a) != all && wrong++ < 10)
                                    std::printf("N %d groups %d pad %d bias %d up %d residual %d Y %d: %d\n", (int)N, groups, (int)pad, bias, up, res, y, (int)!all);
                            }
    if (!wide) std::printf("no case was wide\n");
    return wrong || !wide;
}
"""


def test_whole_accesses_only_where_every_address_is_aligned(tmp_path):
    code, out = host_program.run(tmp_path, PROGRAM)
    assert code == 0, out
