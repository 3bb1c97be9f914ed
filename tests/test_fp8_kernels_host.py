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
            half.add(k16), full.add(k32)
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


def test_choices_at_measured_sizes(kernel):
    """At the sizes that the choices' comments give two times for, the choice is the faster side, or the one launch where
    the two are near."""
    one, two = ((4, 5, 6, 12, 13, 14), (1, 2, 9, 10, 16, 17, 18, 19))
    for M, N, K, fused in ((1, 4096, 4096, True), (1, 8192, 2048, True), (1, 11008, 4096, True), (1, 9000, 6000, False),
                           (1, 8192, 8192, False), (1, 32000, 4096, False), (16, 8192, 2048, True), (16, 4096, 4096, True),
                           (16, 11008, 4096, False), (8, 1024, 8192, True), (16, 1024, 8192, False), (24, 1111, 1000, True), (24, 4096, 4096, False), (32, 1111, 1000, True),
                           (32, 4096, 4096, False), (16, 512, 11008, False), (24, 1024, 4096, False), (1, 1111, 1001, True), (8, 8192, 1004, True),
                           (1, 4096, 2100, False), (8, 4096, 4100, False)):
        assert kernel(0, M, N, K, 0, BF16, BF16) in (one if fused else two), (M, N, K)
    for M, E, N, K, fused in ((64, 8, 4096, 1024, True), (600, 64, 1024, 1024, True), (160, 16, 2048, 2048, True),
                              (64, 8, 5632, 2048, True), (85, 8, 5632, 2048, False), (600, 64, 1408, 2048, False),
                              (128, 16, 1024, 4096, False), (24, 4, 4096, 4096, False), (40, 8, 1024, 8192, False), (6, 8, 2048, 1003, True),
                              (32, 8, 2048, 1003, False), (32, 8, 5632, 2050, False)):
        assert kernel(1, M, N, K, E, BF16, BF16) in (one if fused else two), (M, E, N, K)
    for M, E, N, K, streams in ((16, 8, 4096, 1024, False), (64, 32, 2048, 1024, False), (100, 16, 4096, 1408, True),
                                (32, 8, 5632, 2048, True), (64, 8, 5632, 2048, False), (85, 8, 5632, 2048, False),
                                (100, 16, 2048, 2048, True), (600, 64, 1408, 2048, False), (160, 16, 1024, 4096, True),
                                (40, 4, 4096, 4096, True), (80, 8, 1024, 8192, True)):
        assert (kernel(1, M, N, K, E, 0, BF16) in (1, 9)) == streams, (M, E, N, K)
    for M, N, K, E, wide in ((1, 4096, 4096, 0, False), (16, 8192, 2048, 0, True), (1, 11008, 2048, 0, True), (1, 32000, 1000, 0, True),
                             (1, 11008, 4096, 0, False), (16, 1024, 1024, 8, True), (32, 5632, 2048, 8, True),
                             (24, 4096, 4096, 8, True)):
        assert (kernel(1 if E else 0, M, N, K, E, BF16, BF16) in (5, 13)) == wide, (M, N, K, E)
