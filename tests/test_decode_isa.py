"""What the attention kernel's speed rests on and the compiler decides, read from the assembly of the build (no GPU needed): its
addresses are uniform (a buffer load whose descriptor is not turns into a loop over the lanes), its registers hold the next tile without
spilling, and its loop waits for loads by their count."""
import re

import pytest

from paper_2605_19561_amd import build

# (rows of up to 64 bytes never go past the cache)
# head_dim, MXFP8, past the cache, waves that take turns, products side by side
KERNELS = [(dp, f8, once, ways, rt) for dp in (64, 128, 256) for f8 in (0, 1) for once in (0, 1) for ways in (1, 4) for rt in (1, 2)
           if not (dp == 64 and f8 and once) and not (rt == 2 and (dp == 256 or once and ways == 1))]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    text = open(build.device_asm("paged_attention.hip", str(tmp_path_factory.mktemp("isa") / "a.s"))).read()
    found = {}
    for m in re.finditer(r"^(_ZN4torq22paged_attention_kernelILi(\d+)ELb(\d)ELb(\d)ELi(\d)ELi(\d)E\S*):[^\n]*$(.*?)\.end_amdhsa_kernel", text, re.S | re.M):
        meta = re.search(r"\.name:\s+" + m.group(1) + r"\n(.*?)\.wavefront_size", text, re.S).group(1)
        found[tuple(int(x) for x in m.group(2, 3, 4, 5, 6))] = (m.group(7).split("\n"), meta)
    return found


def loop_of(lines):
    """The innermost loop that holds the products."""
    labels = {m.group(1): i for i, l in enumerate(lines) if (m := re.match(r"^(\.LBB\S+):", l))}
    loops = []
    for i, l in enumerate(lines):
        m = re.search(r"s_c?branch\S*\s+(\.LBB\S+)", l)
        if m and labels.get(m.group(1), i) < i:
            body = lines[labels[m.group(1)]:i]
            if sum("v_mfma" in x for x in body) > 8:
                loops.append(body)
    return min(loops, key=len)


def test_every_attention_kernel_is_there(kernels):
    assert sorted(kernels) == sorted(KERNELS)


@pytest.mark.parametrize("dp,f8,once,ways,rt", KERNELS)
def test_attention_kernel_keeps_its_tile_in_registers_and_its_addresses_uniform(kernels, dp, f8, once, ways, rt):
    lines, meta = kernels[dp, f8, once, ways, rt]
    number = lambda what: int(re.search(r"\." + what + r":\s+(\d+)", meta).group(1))
    assert number("vgpr_spill_count") == 0 and number("private_segment_fixed_size") == 0
    # so many waves fit a SIMD (its 512 registers for each lane) as the launch counts on: three, two or one
    assert number("vgpr_count") <= {64: 168, 128: 256, 256: 512}[dp]
    # a loop over the lanes around a load would branch back right behind it
    for i, l in enumerate(lines):
        if "buffer_load" in l:
            assert not any("s_cbranch_execnz" in x for x in lines[i + 1:i + 4]), lines[i:i + 4]


@pytest.mark.parametrize("dp,f8,once,ways,rt", KERNELS)
def test_attention_loop_waits_by_count(kernels, dp, f8, once, ways, rt):
    loop = loop_of(kernels[dp, f8, once, ways, rt][0])
    loads = [l for l in loop if re.search(r"\b(buffer|global)_load", l)]
    k, v = 2 * dp * (1 if f8 else 2) // 64, 8 * (2 if dp == 256 else 1)
    assert len(loads) == (k + v) * (2 if f8 else 1)                          # K and V of the next tile, and their scales
    assert sum(" nt" in l for l in loads) == ((k + v) if once else 0)        # (the scales' lines are shared)
    # the wait for this tile's K leaves V's loads on their way
    counts = [int(m.group(1)) for l in loop if (m := re.search(r"s_waitcnt.*vmcnt\((\d+)\)", l))]
    assert counts and min(counts) > 0, counts
