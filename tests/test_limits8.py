"""Sizes that one launch of the 8-bit path cannot take (fewer than 2^32 threads) are refused before anything is enqueued; no call
here reaches a device."""
import pytest

from paper_2608_24070_amd import slim

A = 1 << 20          # a fake, 16-byte aligned, non-null "device" address (never dereferenced)
F16, F32, Q8 = slim.SLIM_F16, slim.SLIM_F32, slim.SLIM_Q8_E4M3


@pytest.mark.parametrize("k,xdt", [(8193, F32), (16383, F32), (8193, Q8), (12001, Q8)])
def test_fp32_rows_that_end_inside_a_vector(k, xdt):
    # a block of 1024 threads a row in the backward's second launch
    m = 1 << 22
    need = slim.slim_norm_bwd_workspace(m, k)
    assert slim.slim_norm_bwd(A, F32, k, A, xdt, A, k, m, k, None, F32, A, A, A, k, A, A, A, need, None) == slim.SLIM_EUNSUPPORTED
