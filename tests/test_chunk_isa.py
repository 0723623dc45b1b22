"""What the compiler makes of the prompt attention's kernels of 256 rows: O lies in the accumulators' half from a128 on, by name, and what the kernels' own
statements leave to the compiler there has to hold in the code that it makes."""
import concurrent.futures
import re

import pytest

from paper_2605_19561_amd.build import device_asm

SOURCES = ["chunk_attention_64.hip", "chunk_attention_96.hip", "chunk_attention_128.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: text} of the kernels whose waves have two blocks of rows."""
    folder = tmp_path_factory.mktemp("asm")
    with concurrent.futures.ThreadPoolExecutor(3) as pool:
        texts = [open(f).read() for f in pool.map(lambda s: device_asm(s, str(folder / (s + ".s"))), SOURCES)]
    found = {m[1]: m[2] for t in texts
             for m in re.finditer(r"^(_ZN4torq22chunk_attention_kernel\S*ELi4ELi2EEEv\S*):[^\n]*$(.*?)\.end_amdhsa_kernel", t, re.S | re.M)}
    assert len(found) == 3 * 3 * 2                    # widths, formats, with and without slopes
    return found


def registers(operand, half):
    m = re.match(r"%s(?:\[(\d+):(\d+)\]|(\d+))$" % half, operand.strip())
    return set() if not m else {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def code(text):
    lines = [re.sub(r";.*", "", l).strip() for l in text.split("\n")]
    return [l for l in lines if l and not l.startswith(".")]


def test_the_compiler_leaves_o_alone(kernels):
    for name, text in kernels.items():
        rest = re.sub(r";+#ASMSTART.*?;+#ASMEND", "", text, flags=re.S)
        for line in code(rest):
            used = [int(x) for m in re.findall(r"\ba(?:\[(\d+):(\d+)\]|(\d+))", line) for x in m if x]
            assert not used or max(used) < 128, (name, line)


def test_no_operand_of_o_is_written_just_ahead_of_its_product(kernels):
    """A vector instruction's result may be a product's operand two wait states later, which the compiler does not look after in such statements."""
    for name, text in kernels.items():
        lines, products = code(text), 0
        for i, line in enumerate(lines):
            if not re.match(r"v_mfma\S+\s+a\[\w+:\w+\+15\]", line):        # (as the statement is written)
                continue
            products += 1
            operands = line.split(None, 1)[1].split(",")
            read, waits, j = registers(operands[1], "v") | registers(operands[2], "v"), 0, i - 1
            assert len(read) == 8
            while waits < 2:
                before, j = lines[j], j - 1
                if before.startswith("s_nop"):
                    waits += int(before.split()[1]) + 1
                    continue
                if before.startswith("v_") and not before.startswith("v_mfma"):
                    assert not read & registers(before.split(None, 1)[1].split(",")[0], "v"), (name, before, line)
                waits += 1
        assert products >= 16, name


def test_nothing_is_spilled(kernels):
    for name, text in kernels.items():
        assert "scratch_" not in "\n".join(code(text)), name
