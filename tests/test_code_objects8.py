"""What the compiler made of the 8-bit products whose matrix instructions and LDS reads are written out."""
import os
import re

import pytest

from paper_2608_24070_amd import slim
from tests import code_objects
from tests.test_code_objects import touched_in_flight


def sums_read_early(body):
    """Instructions other than products that name an accumulation register with fewer than 16 wait states since the last
    product before them: a written-out product is no product to the compiler, which adds no wait states after it."""
    bad, since = [], None
    for at, text in body:
        op, _, rest = text.partition(" ")
        if op.startswith("v_mfma"):
            since = 0
            continue
        if since is not None and since < 16 and re.search(r"\ba\[?\d", rest) and not op.startswith("v_accvgpr_write"):
            bad.append((at, text))
        if since is not None and op == "s_nop":
            since += int(rest, 0) + 1
    return bad


def test_sums_read_early_sees_a_missing_wait():
    ok = [(0, "v_accvgpr_write_b32 a0, v1"), (8, "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]"), (16, "s_nop 15"),
          (20, "v_accvgpr_read_b32 v0, a0"), (28, "ds_write_b64 v1, a[2:3]")]
    assert not sums_read_early(ok)
    assert sums_read_early(ok[:2] + ok[3:]) == ok[3:]
    assert sums_read_early(ok[:2] + [(16, "s_nop 7")] + ok[3:]) == ok[3:]


@pytest.fixture(scope="module")
def bodies(tmp_path_factory):
    if not os.path.exists(code_objects.OBJDUMP):
        pytest.skip("no llvm-objdump")
    all_ = code_objects.disassembly(slim.LIB_PATH, str(tmp_path_factory.mktemp("objects")))
    found = {n: b for n, b in all_.items() if re.search(r"\d(k_linear8_tileI|k_wgrad8_wideI)", n) and not n.endswith(".kd")}
    # six tiles for two types of result; two types of dY, whole or at kept positions
    assert sum("k_linear8_tile" in n for n in found) == 12 and sum("k_wgrad8_wide" in n for n in found) >= 2, sorted(found)
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
    # no move between accumulation registers and others inside the loop, from its first product to its last
    for n, body in bodies.items():
        at = [i for i, (_, t) in enumerate(body) if t.startswith("v_mfma")]
        moves = [t for _, t in body[at[0]:at[-1]] if t.startswith("v_accvgpr")]
        assert not moves, (n, moves[:4])
