"""Which kernel a product of 8-bit floats takes (no GPU: the choice goes by 256 compute units there, as on an MI355X)."""
import os

import pytest

import _fp8_cases as cases

F16, BF16, I8, F32 = 1, 2, 3, 5


@pytest.fixture(scope="module")
def kernel():
    from paper_2405_03594_amd import LIB_PATH, build

    if not os.path.exists(LIB_PATH):
        build.build()
    import paper_2405_03594_amd as spl

    return spl.lib().spl_linear_fp8_kernel


def test_cases_reach_their_kernels(kernel):
    """Every case of the GPU tests takes the kernel that it stands for, and no kernel is without one."""
    wrong, half, full = [], set(), set()

    def check(case, got, want):
        if got != want:
            wrong.append((case, got, want))

    for table, x in ((cases.CODES, (0,)), (cases.ROWS, (F16, BF16))):
        for M, N, K, k16, k32 in table:
            for t in x:
                for d, want in ((F16, k16), (BF16, k16), (F32, k32)):
                    check((M, N, K, t, d), kernel(0, M, N, K, 0, t, d), want)
            half.add(k16), full.add(k32)
    for starts, M, N, K, c16, c32, r16, r32 in cases.GROUPED:
        for t, k16, k32 in ((0, c16, c32), (F16, r16, r32), (BF16, r16, r32)):
            for d, want in ((F16, k16), (BF16, k16), (F32, k32)):
                check((len(starts) - 1, M, N, K, t, d), kernel(1, M, N, K, len(starts) - 1, t, d), want)
    for starts, M, N, T, k16, k32 in cases.SUMS:
        for d, want in ((F16, k16), (BF16, k16), (F32, k32)):
            check((len(starts) - 1, M, N, T, d), kernel(2, M, N, T, len(starts) - 1, 0, d), want)
    assert not wrong, wrong
    assert half == cases.EVERY - {21}
    assert full == cases.EVERY - {18, 19, 20}
    assert {r for g in cases.GROUPED for r in g[4:]} >= {1, 9, 4, 5, 13, 16, 17, 18, 19, 21}


def test_refused_sizes(kernel):
    for args in ((3, 1, 1, 1, 1, 0, BF16), (-1, 1, 1, 1, 1, 0, BF16), (0, 0, 1, 1, 1, 0, BF16), (0, 1, 0, 1, 1, 0, BF16),
                 (0, 1, 1, 0, 1, 0, BF16), (0, 1, 1, 1, 1, F32, BF16), (0, 1, 1, 1, 1, 0, I8), (1, 1, 1, 1, 0, 0, BF16),
                 (2, 1, 1, 1, 0, 0, F32), (2, 1, 1, 1, 1, BF16, F32), (0, 1 << 31, 1, 1, 1, 0, BF16), (0, 1, 1, 1 << 23, 1, 0, F32),
                 (1, (1 << 22) + 1, 1, 1, 1, 0, BF16), (2, 1, 1, (1 << 22) + 1, 1, 0, F32)):
        assert kernel(*args) == -1, args


def test_workspace_goes_with_the_kernel(kernel):
    """Scratch memory for the sums of codes is asked for where they are split, and only there."""
    import paper_2405_03594_amd as spl

    need = spl.lib().spl_linear_fp8_workspace_bytes
    for M, N, K, k16, k32 in cases.CODES:
        assert (need(M, N, K) > 0) == (k16 == 22) == (k32 == 22), (M, N, K)
        if k16 == 22:
            assert need(M, N, K) >= 2 * 4 * M * N and need(M, N, K) % 256 == 0
