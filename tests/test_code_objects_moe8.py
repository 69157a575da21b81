"""What the compiler made of the experts' products: no result of a matrix instruction is read before it is written. The hardware does
not wait there; the compiler counts instructions, but not along every way past a branch."""
import os
import re

import pytest

from paper_2608_24070_amd import slim
from tests import code_objects

# wait states that the compiler puts between a product of 16 x 16 x 32 and another kind of instruction that reads it next
NEED = 8


def registers(text):
    out = set()
    for kind, lo, hi in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {kind + str(r) for r in range(int(lo), int(hi) + 1)}
    return out | {k + r for k, r in re.findall(r"\b([va])(\d+)\b", text)}


def read_early(body):
    """(product, reader) pairs with fewer than NEED wait states between them on some path."""
    where, bad = {at: i for i, (at, _) in enumerate(body)}, set()
    for i0, (at0, text0) in enumerate(body):
        if not text0.startswith("v_mfma"):
            continue
        dest = registers(text0.split(None, 1)[1].split(",")[0])
        work, seen = [(i0 + 1, 0)], set()
        while work:
            i, states = work.pop()
            while i < len(body) and states < NEED and (i, states) not in seen:
                seen.add((i, states))
                at, text = body[i]
                op = text.split(None, 1)[0]
                if op.startswith("v_mfma"):
                    if registers(text.split(None, 1)[1].split(",")[0]) & dest:
                        break                       # the sum goes on; its own reads are looked at from there
                    states += 4                     # a matrix instruction keeps the next one waiting at least so long
                elif op == "s_nop":
                    states += int(text.split()[1], 0) + 1
                elif op == "s_endpgm":
                    break
                elif op.startswith(("s_cbranch", "s_branch")):
                    off = int(text.split()[1])
                    target = where.get(at + 4 + 4 * (off - 65536 if off >= 32768 else off))
                    if op == "s_branch":
                        if target is None:
                            break
                        i, states = target, states + 1
                        continue
                    if target is not None:
                        work.append((target, states + 1))
                    states += 1
                else:
                    if registers(text) & dest:
                        bad.add((text0, text))
                        break
                    states += 1
                i += 1
    return bad


def test_read_early_sees_a_way_past_a_branch():
    ok = [(0, "v_mfma_f32_16x16x32_bf16 v[8:11], v[0:3], v[4:7], 0"), (8, "s_cbranch_vccnz 3"), (12, "s_nop 15"), (16, "s_nop 0"),
          (20, "s_nop 0"), (24, "v_fmac_f32_e32 v20, v8, v21"), (28, "s_endpgm")]
    assert read_early(ok)
    assert not read_early([ok[0], (8, "s_nop 0")] + ok[2:])
    far = [ok[0], (8, "s_nop 15"), (12, "v_fmac_f32_e32 v20, v8, v21"), (16, "s_endpgm")]
    assert not read_early(far)


@pytest.mark.skipif(not os.path.exists(code_objects.OBJDUMP), reason="no llvm-objdump")
def test_products_are_written_before_they_are_read(tmp_path):
    bodies = code_objects.disassembly(slim.LIB_PATH, str(tmp_path))
    names = [n for n in bodies if re.search(r"\dk_(moe_up|moe_down|act8_few)I", n) and not n.endswith(".kd")]
    assert len(names) >= 3 * 2 + 2 + 6, names
    for n in names:
        assert sum(t.startswith("v_mfma") for _, t in bodies[n]) >= 4, n
        assert not read_early(bodies[n]), (n, sorted(read_early(bodies[n]))[:3])
