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


@pytest.mark.parametrize("m,n,k", [(1 << 22, 1 << 20, 128), (1 << 21, 1 << 22, 100)])
def test_tiles_of_the_product(m, n, k):
    # 256 x 256 tiles of 256 threads
    with pytest.raises(slim.SlimError) as e:
        slim.slim_linear8_workspace(Q8, m, n, k)
    assert e.value.status == slim.SLIM_EUNSUPPORTED
    assert slim.slim_linear8(A, Q8, A, m, n, k, 0, A, A, A, F16, n, A, 1 << 40, None) == slim.SLIM_EUNSUPPORTED


@pytest.mark.parametrize("m,n,k,masked", [(64, 1 << 20, 1 << 18, 0), (0, 1 << 20, 1 << 20, 1), (1000, 1 << 22, 1 << 22, 0)])
def test_tiles_of_the_weight_gradient(m, n, k, masked):
    # 128 x 128 tiles of 512 threads, or 256 x 256 of 256
    with pytest.raises(slim.SlimError) as e:
        slim.slim_grad_w8_workspace(m, n, k, masked, 1)
    assert e.value.status == slim.SLIM_EUNSUPPORTED
    assert slim.slim_grad_w8(A, F16, n, A, A, m, n, k, A if masked else None, A, A, 1 << 50, None) == slim.SLIM_EUNSUPPORTED


def test_the_largest_that_are_taken():
    assert slim.slim_linear8_workspace(Q8, 1 << 21, 1 << 17, 128) == 0 and slim.slim_linear8_workspace(Q8, 1 << 14, 1 << 22, 28672) == 0
    assert slim.slim_grad_w8_workspace(8192, 1 << 19, 1 << 19, 0, 1) == 0 and slim.slim_grad_w8_workspace(64, 1 << 18, 1 << 18, 0, 1) == 0
