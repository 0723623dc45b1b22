"""The attention kernel's two forms, a workgroup for each (request, key head) and equal runs of tiles, in the assembly of the build (no GPU
needed): each keeps what its speed rests on, and the first carries nothing of the second's."""
import re

import pytest

from paper_2605_19561_amd import build
from test_decode_isa import KERNELS, loop_of

FORMS = [(*k, solo) for k in KERNELS for solo in (0, 1)]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    text = open(build.device_asm("paged_attention.hip", str(tmp_path_factory.mktemp("isa") / "a.s"))).read()
    found = {}
    for m in re.finditer(r"^(_ZN4torq22paged_attention_kernelILi(\d+)ELb(\d)ELb(\d)ELi(\d)ELi(\d)ELb(\d)E\S*):[^\n]*$(.*?)\.end_amdhsa_kernel", text, re.S | re.M):
        meta = re.search(r"\.name:\s+" + m.group(1) + r"\n(.*?)\.wavefront_size", text, re.S).group(1)
        found[tuple(int(x) for x in m.group(2, 3, 4, 5, 6, 7))] = (m.group(8).split("\n"), meta)
    return found


def test_every_kernel_is_there_in_both_forms(kernels):
    assert sorted(kernels) == sorted(FORMS)


@pytest.mark.parametrize("dp,f8,once,ways,rt,solo", FORMS)
def test_both_forms_keep_their_tile_in_registers_and_wait_by_count(kernels, dp, f8, once, ways, rt, solo):
    lines, meta = kernels[dp, f8, once, ways, rt, solo]
    number = lambda what: int(re.search(r"\." + what + r":\s+(\d+)", meta).group(1))
    assert number("vgpr_spill_count") == 0 and number("private_segment_fixed_size") == 0
    assert number("vgpr_count") <= {64: 168, 128: 256, 256: 512}[dp]
    for i, l in enumerate(lines):
        if "buffer_load" in l:
            assert not any("s_cbranch_execnz" in x for x in lines[i + 1:i + 4]), lines[i:i + 4]
    loop = loop_of(lines)
    loads = [l for l in loop if re.search(r"\b(buffer|global)_load", l)]
    k, v = 2 * dp * (1 if f8 else 2) // 64, 8 * (2 if dp == 256 else 1)
    assert len(loads) == (k + v) * (2 if f8 else 1)
    assert sum(" nt" in l for l in loads) == ((k + v) if once else 0)
    counts = [int(m.group(1)) for l in loop if (m := re.search(r"s_waitcnt.*vmcnt\((\d+)\)", l))]
    assert counts and min(counts) > 0, counts


@pytest.mark.parametrize("dp,f8,once,ways,rt", KERNELS)
def test_a_workgroup_for_each_column_carries_nothing_of_the_runs(kernels, dp, f8, once, ways, rt):
    # sums over the requests (DPP adds across rows), the lane that a run begins in (a ballot's first bit), the next request's tiles
    text = {solo: "\n".join(kernels[dp, f8, once, ways, rt, solo][0]) for solo in (0, 1)}
    for sign in (r"row_bcast", r"s_ff1_i32_b64|s_ff1_i32_b32"):
        assert re.search(sign, text[0]) and not re.search(sign, text[1]), sign
    assert len(text[1]) < len(text[0])
