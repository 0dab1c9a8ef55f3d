"""Which kernel an MX4 product takes, on the host: the sizes that stand for each kernel really take it."""
import pytest

import paper_2508_19087_amd as apt
from mx_sizes import FUSED, KERNELS, TURN


def block(M, N, K):
    st, rows, columns = apt.apt_mx4_select(M, N, K)
    assert st == apt.APT_OK
    return rows, columns


@pytest.mark.parametrize("kernel", KERNELS)
def test_sizes_take_their_kernel(kernel):
    for s in KERNELS[kernel]:
        assert block(*s) == kernel, s


@pytest.mark.parametrize("kernel", KERNELS)
def test_sizes_leave_every_rest(kernel):
    """Tiles: every number of steps behind the last four, with and without a further turn before, and one
    to three steps alone (the largest is taken for long K only).  Few rows: waves that share a turn's
    rest evenly and not."""
    turn, steps = TURN[kernel], {-(-K // 256) for _, _, K in KERNELS[kernel]}
    if turn == 4:
        assert {s % 4 for s in steps if s > 4} == {0, 1, 2, 3}
        assert kernel == (256, 256) or {1, 2, 3, 4} <= steps
    else:
        rests = {(s % turn // 4, s % 4 != 0) for s in steps if s > turn}
        assert rests == {(i, j) for i in range(turn // 4) for j in (False, True)}
        assert kernel in ((32, 32), (64, 32)) or {1, 2, 3, 4} <= steps
    for M, N, K in KERNELS[kernel]:
        assert M % kernel[0] and N % kernel[1] and K % 32


def test_few_rows_never_take_tiles():
    for M in range(1, 33):
        for N in (1, 100, 5000, 30000):
            for K in (1, 1000, 11008):
                assert block(M, N, K)[1] <= 32
    for M in range(1, 17):
        assert block(M, 11008, 4096) == (16, 16)  # the kernel that quantizes rows itself: the same sums


def test_rows_that_the_product_quantizes():
    assert {s[0] for s in FUSED} == set(range(1, 17))
    for s in FUSED:
        assert apt.apt_mx4_gemm_act_workspace_bytes(*s) == 0, s
        # (the longest rows that are taken)
        M, N, _ = s
        most = 64 // M * 256
        assert apt.apt_mx4_gemm_act_workspace_bytes(M, N, most) == 0
        assert apt.apt_mx4_gemm_act_workspace_bytes(M, N, most + 1) == apt.apt_mx4_bytes(M, most + 1)
    assert apt.apt_mx4_gemm_act_workspace_bytes(17, 5, 1) == apt.apt_mx4_bytes(17, 1)


@pytest.mark.parametrize("bad", [(0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1), (2 ** 31, 1, 1)])
def test_select_refuses(bad):
    assert apt.apt_mx4_select(*bad)[0] == apt.APT_ERR_INVALID_ARG


def test_select_limits():
    for s in ((1, 1, 2 ** 24 + 1), (2 ** 31 - 1, 1, 1), (1, 2 ** 31 - 1, 257), (2 ** 27, 2 ** 27, 1)):
        assert apt.apt_mx4_select(*s)[0] == apt.APT_ERR_UNSUPPORTED
    assert apt.lib().apt_mx4_select(1, 1, 1, None, None) == apt.APT_ERR_INVALID_ARG


@pytest.mark.parametrize("M,K,most", [(3, 4096, 21840), (4, 4096, 16384), (16, 1024, 16384), (8, 1024, 32768), (3, 256, 349520)])
def test_rows_are_quantized_once_where_many_weight_rows_repeat_it(M, K, most):
    """Up to 2^24 elements times groups of 16 weight rows, from three rows on."""
    assert apt.apt_mx4_gemm_act_workspace_bytes(M, most, K) == 0
    assert apt.apt_mx4_gemm_act_workspace_bytes(M, most + 1, K) == apt.apt_mx4_bytes(M, K)
    for rows in (1, 2):
        assert apt.apt_mx4_gemm_act_workspace_bytes(rows, 128000, K) == 0
