"""What the compiler made of the products that end in an activation: the loop's matrix instructions and LDS reads are written out."""
import os
import re

import pytest

from paper_2608_24070_amd import slim
from tests import code_objects
from tests.test_code_objects import touched_in_flight
from tests.test_code_objects8 import sums_read_early


@pytest.fixture(scope="module")
def bodies(tmp_path_factory):
    if not os.path.exists(code_objects.OBJDUMP):
        pytest.skip("no llvm-objdump")
    all_ = code_objects.disassembly(slim.LIB_PATH, str(tmp_path_factory.mktemp("objects")))
    found = {n: b for n, b in all_.items() if re.search(r"\dk_act8_tileI", n) and not n.endswith(".kd")}
    # five tiles forward and backward for two types, three that leave sums
    assert len(found) == 23, sorted(found)
    return found


def test_written_out_reads_land_before_their_registers_are_used(bodies):
    for n, body in bodies.items():
        assert sum(t.startswith("ds_read") for _, t in body) > 16, n
        assert not touched_in_flight(body), n


def test_sums_are_read_after_the_last_product_is_written(bodies):
    for n, body in bodies.items():
        assert sum(t.startswith("v_mfma") for _, t in body) >= 64, n
        assert not sums_read_early(body), n


def test_sums_stay_in_their_registers(bodies):
    for n, body in bodies.items():
        at = [i for i, (_, t) in enumerate(body) if t.startswith("v_mfma")]
        moves = [t for _, t in body[at[0]:at[-1]] if t.startswith("v_accvgpr")]
        assert not moves, (n, moves[:4])
