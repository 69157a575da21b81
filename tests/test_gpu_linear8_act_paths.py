"""The paths of the products that end in an activation which the sizes of test_gpu_linear8_act do not reach: 128 x 128 tiles in slices of
the reduction, and 64-column tiles over the whole of it, both by fp32 sums in memory. The same checks and bounds."""
import pytest

from tests import test_gpu_linear8_act as t

pytestmark = pytest.mark.gpu

# 128 x 128 tiles in four slices; 64-column tiles over the whole reduction
SIZES = [(715, 1071, 10244), (1024, 770, 20001), (1689, 526, 10140), (2985, 261, 8005)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_forward(m, n, k):
    t.test_forward(m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_nothing_added_is_the_product(m, n, k):
    t.test_nothing_added_is_the_product(m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_backward(m, n, k):
    t.test_backward(m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES[1:3])
def test_repeats_streams_and_graph_replays(m, n, k):
    t.test_repeats_streams_and_graph_replays(m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_workspaces_are_what_is_asked_for(m, n, k):
    t.test_workspaces_are_what_is_asked_for(m, n, k)
