"""The sizes from which on the router and the experts return SLIM_EUNSUPPORTED, where the header puts them (host only)."""
import pytest

from paper_2608_24070_amd import slim

A = 1 << 20          # never dereferenced


def refused(query, *args):
    with pytest.raises(slim.SlimError) as e:
        query(*args)
    return e.value.status == slim.SLIM_EUNSUPPORTED


def test_route_rows():
    # the choice's launch, a wave a row: it binds where experts and columns are few
    most = (1 << 26) - 4
    for e, k in ((1, 256), (3, 2048)):
        assert slim.slim_route_workspace(most, e, k) == most * e * 4 and refused(slim.slim_route_workspace, most + 1, e, k)
    assert refused(slim.slim_route_workspace, 1 << 27, 1, 256)
    assert slim.slim_route(A, slim.SLIM_BF16, None, 1 << 27, 256, 256, A, slim.SLIM_F32, 1, 256, 1, 1, A, A, A, 1 << 62, None) == slim.SLIM_EUNSUPPORTED


def test_route_blocks():
    # the logits' launch: 16 rows, 2048 columns, an expert
    for e, k in ((40, 256), (512, 8192), (4, 2049)):
        most = ((1 << 24) - 1) // (e * -(-k // 2048)) * 16
        assert slim.slim_route_workspace(most, e, k) > 0 and refused(slim.slim_route_workspace, most + 1, e, k)


def test_experts_columns():
    most = (1 << 19) - 128
    assert slim.slim_moe8_workspace(64, 128, most, 512, 16) > 0 and refused(slim.slim_moe8_workspace, 64, 128, most + 1, 512, 16)
    # by the experts that rows may pick, not by those that are there
    assert slim.slim_moe8_workspace(1, 128, 1 << 22, 512, 16) > 0 and slim.slim_moe8_workspace(4, 128, 1 << 21, 512, 16) > 0
    assert refused(slim.slim_moe8_workspace, 64, 128, 1 << 22, 512, 16)
