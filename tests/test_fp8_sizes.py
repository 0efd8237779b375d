"""Sizes that the 8-bit floating-point linears refuse, asked for their workspace."""
import pytest

from paper_2503_06545_amd import binding as qc


@pytest.mark.parametrize("M,K,N", [(1 << 31, 8, 8), (1 << 30, 9216, 8), (1 << 40, 1152, 1152), (1 << 62, qc.QC_MAX_K, 8), (2 ** 63 - 1, 1, 1),
                                   (8, 8, qc.QC_MAX_N + 1), (1 << 29, 128, 1)])
def test_sizes_that_the_linear_refuses_have_no_workspace(M, K, N):
    """Not the size of a product that has wrapped round, nor gigabytes for a call that cannot be made.  (2^29 rows are 2^24 blocks of 32
    rows and 256 threads for each 128 columns, 2^32 threads, one more than a launch can have.)"""
    A = 0x10000   # never dereferenced
    assert qc.qc_qlinear_fp8(A, qc.QC_BF16, M, K, A, A, N, None, qc.QC_EPI_NONE, A, qc.QC_OUT_BF16, A, 2 ** 63 - 1) == qc.QC_ERR_UNSUPPORTED
    assert qc.qc_qlinear_fp8_workspace_bytes(M, K, N) == 0
    with pytest.raises(qc.QcError):
        qc.qlinear_fp8_workspace_t(M, K, N)


def test_the_largest_that_it_takes_have_one():
    for M, K, N in ((1 << 28, 128, 1), ((1 << 29) - 1024, 128, 1), (1, qc.QC_MAX_K, qc.QC_MAX_N), (1, 1, 1)):
        assert qc.qc_qlinear_fp8_workspace_bytes(M, K, N) >= M * K
