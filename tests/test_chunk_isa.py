"""What the kernels for prompts, for caches in MXFP4 and for scores by a rule rest on and the compiler decides, read from the assembly of the build (no GPU
needed): registers for the waves that a launch counts on, addresses that are uniform, and in the loop over bf16 the waits, which count by hand the loads that are
on their way into LDS."""
import concurrent.futures
import re

import pytest

from paper_2605_19561_amd import build

BF16, MXFP8, MXFP4 = 8, 9, 0
PLAIN, CAP, SLOPES, ANY = range(4)                   # what is done to scores
# values of a row in LDS, those that are multiplied
WIDTHS = [(64, 64), (128, 96), (128, 128), (256, 192), (256, 256)]
# ..., format, scores, waves that share keys
CHUNKS = [(dp, dv, fmt, bend, rw) for dp, dv in WIDTHS for fmt in (BF16, MXFP8, MXFP4) for bend in range(4) for rw in (2, 4) if dp < 256 or rw == 4]
# bytes of scratch that are accepted: a register or some, put away and taken back in each step of kernels that have all 512
SCRATCH = {(256, 256, MXFP8, PLAIN, 4): 8, (256, 256, MXFP4, PLAIN, 4): 20}
# head_dim, past the cache, waves that take turns, products side by side, a workgroup each
FOURS = [(dp, once, ways, rt, solo) for dp in (64, 128, 256) for once in (0, 1) for ways in (1, 4) for rt in (1, 2) for solo in (0, 1)
         if not (once and dp < 256) and not (rt == 2 and dp == 256)]
RULED = [(dp, fmt, once, ways, rt, solo) for dp in (64, 128, 256) for fmt, bits in ((BF16, 16), (MXFP8, 8), (MXFP4, 4)) for once in (0, 1) for ways in (1, 4)
         for rt in (1, 2) for solo in (0, 1) if not (once and dp * bits < 1024) and not (rt == 2 and (dp == 256 or once and ways == 1))]
SOURCES = {"chunk_attention_kernel": ["chunk_attention_%d.hip" % n for n in (64, 96, 128, 192, 256)],
           "paged_attention4_kernel": ["paged_attention_mxfp4.hip"],
           "scored_attention_kernel": ["paged_attention_scores_%s.hip" % f for f in ("bf16", "mxfp8", "mxfp4")]}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: {its template's numbers: (lines, what is said of it)}}"""
    folder = tmp_path_factory.mktemp("isa")
    names = [s for sources in SOURCES.values() for s in sources]
    with concurrent.futures.ThreadPoolExecutor(8) as pool:
        texts = dict(zip(names, pool.map(lambda s: open(build.device_asm(s, str(folder / (s + ".s")))).read(), names)))
    found = {kernel: {} for kernel in SOURCES}
    for kernel, sources in SOURCES.items():
        for text in (texts[s] for s in sources):
            said = dict(re.findall(r"\.name:\s+(\S+)\n(.*?)\.wavefront_size", text, re.S))
            for m in re.finditer(r"^(_ZN4torq%d%sI(\S*?)EEvNS_\S*):[^\n]*$(.*?)\.end_amdhsa_kernel" % (len(kernel), kernel), text, re.S | re.M):
                found[kernel][tuple(int(x) for x in re.findall(r"L[ib](\d+)E", m[2] + "E"))] = (m[3].split("\n"), said[m[1]])
    return found


def number(said, what):
    return int(re.search(r"\." + what + r":\s+(\d+)", said)[1])


def test_every_kernel_is_there(kernels):
    assert sorted(kernels["chunk_attention_kernel"]) == sorted(CHUNKS)
    assert sorted(kernels["paged_attention4_kernel"]) == sorted(FOURS)
    assert sorted(kernels["scored_attention_kernel"]) == sorted(RULED)


def one_load_at_a_time(lines):
    """A load whose descriptor is not the same in every lane: a loop over the lanes branches back right behind it."""
    return [lines[i:i + 4] for i, l in enumerate(lines) if "buffer_load" in l and any("s_cbranch_execnz" in x for x in lines[i + 1:i + 4])]


def test_registers_of_the_prompts_kernels(kernels):
    for at, (lines, said) in kernels["chunk_attention_kernel"].items():
        dp, _, _, _, rw = at
        # two workgroups on a CU, so two waves on a SIMD, or one
        assert number(said, "vgpr_count") <= (256 if dp * (4 // rw) <= 128 else 512), at
        assert number(said, "private_segment_fixed_size") <= SCRATCH.get(at, 0), at
        assert not one_load_at_a_time(lines), at


@pytest.mark.parametrize("kernel", ["paged_attention4_kernel", "scored_attention_kernel"])
def test_registers_of_the_single_tokens_kernels(kernels, kernel):
    for at, (lines, said) in kernels[kernel].items():
        ruled = kernel == "scored_attention_kernel"
        # three, two or one wave on a SIMD; a rule's masks and positions beside two products take one fewer
        assert number(said, "vgpr_count") <= {64: 168, 128: 256, 256: 512}[at[0] * (2 if ruled and at[4] == 2 else 1)], at
        assert number(said, "private_segment_fixed_size") == 0 and number(said, "vgpr_spill_count") == 0, at
        assert not one_load_at_a_time(lines), at


def steps_of(lines):
    """(loads into LDS, waits written by hand) between one barrier and the next."""
    steps, loads, waits, by_hand = [], 0, [], False
    for l in lines:
        by_hand = "#ASMSTART" in l or (by_hand and "#ASMEND" not in l)
        loads += bool(re.search(r"buffer_load\S*\s.*\blds\b", l))
        if by_hand and (m := re.search(r"s_waitcnt vmcnt\((\d+)\)", l)):
            waits.append(int(m[1]))
        if "s_barrier" in l:
            steps.append((loads, waits))
            loads, waits = 0, []
    return steps


@pytest.mark.parametrize("dp,dv,fmt,bend,rw", [at for at in CHUNKS if at[2] == BF16])
def test_prompts_over_bf16_wait_for_all_loads_but_their_steps_own(kernels, dp, dv, fmt, bend, rw):
    steps = steps_of(kernels["chunk_attention_kernel"][dp, dv, fmt, bend, rw][0])
    each = dp // (16 * rw)                           # a wave's loads of 32 / rw keys, 1024 bytes each
    # three steps of K and two of V ahead, all of them there; then K and V of a step, which may still be on their way when those of the step before are there
    assert steps[0] == (5 * each, [0])
    loop = [s for s in steps[1:] if s[0]]
    assert loop == [(2 * each, [2 * each])] * 4      # the first, two by turns, an odd last
    # and none is on its way when LDS becomes the output's
    assert steps[1:5] == loop and steps[5] == (0, [0])
