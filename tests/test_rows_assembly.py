"""What the compiler makes of rows.hip: it inserts the wait states that the hardware leaves to software between instructions
that it knows, not in front of, inside or behind assembly text."""
import os
import re
import subprocess

import pytest

from paper_2512_22219_amd import build as B


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Kernel name -> its assembly, a list of lines."""
    out = str(tmp_path_factory.mktemp("asm") / "rows.s")
    source = next(s for s in B.SOURCES if os.path.basename(s) == "rows.hip")
    subprocess.run(["hipcc", *B.FLAGS, "-S", "--offload-device-only", source, "-o", out], check=True, stderr=subprocess.DEVNULL)
    with open(out) as f:
        bodies = re.findall(r"^(_ZN3mpk\w+):[^\n]*\n(.*?)^\.Lfunc_end", f.read(), re.S | re.M)
    assert sum("rows_attend_kernel" in name for name, _ in bodies) == 8 and sum("rows_logprobs_kernel" in name for name, _ in bodies) == 4
    return {name: body.splitlines() for name, body in bodies}


def _texts(lines):
    """The instructions of each piece of assembly text."""
    texts, inside = [], None
    for line in lines:
        if "#ASMSTART" in line:
            inside = []
        elif "#ASMEND" in line:
            texts.append(inside)
            inside = None
        elif inside is not None:
            inside.append(line.split(";")[0].strip())
    return [[i for i in t if i] for t in texts]


def test_no_vector_operation_is_assembly_text(kernels):
    """A vector operation that reads what a matrix instruction or another lane's has just written needs wait states."""
    for name, lines in kernels.items():
        for text in _texts(lines):
            assert not [i for i in text if i.startswith("v_")], (name, text)


def test_results_of_matrix_instructions_are_waited_for_on_every_path(kernels):
    """From each matrix instruction of 8 passes forward, over branches too: no vector operation reads its results within 12 wait
    states (an instruction is one, s_nop n is n + 1)."""
    registers = lambda x: {int(r) for lo, hi in re.findall(r"\bv\[(\d+):(\d+)\]", x) for r in range(int(lo), int(hi) + 1)} | \
        {int(r) for r in re.findall(r"\bv(\d+)\b", x)}  # noqa: E731
    checked = 0
    for name, lines in kernels.items():
        code, labels = [], {}
        for line in lines:
            if re.match(r"\.L\w+:", line):
                labels[line.split(":")[0]] = len(code)
            line = line.split(";")[0].strip()
            if line and not line.startswith(".") and not line.endswith(":"):
                code.append(line)
        for at, line in enumerate(code):
            m = re.match(r"v_mfma_f32_32x32x16_bf16 (v\[\d+:\d+\])", line)
            if not m:
                continue
            checked += 1
            results, todo, seen = registers(m.group(1)), [(at + 1, 0)], {}
            while todo:
                i, waited = todo.pop()
                if waited >= 12 or i >= len(code) or seen.get(i, 99) <= waited:
                    continue
                seen[i] = waited
                op = code[i].split()[0]
                if op.startswith("v_") and not op.startswith("v_mfma"):
                    assert not results & registers(code[i]), (name, line, code[i], waited)
                after = waited + (int(code[i].split()[1]) + 1 if op == "s_nop" else 1)
                if op.startswith(("s_branch", "s_cbranch")):
                    todo.append((labels[code[i].split()[1]], after))
                if op not in ("s_branch", "s_endpgm"):
                    todo.append((i + 1, after))
    assert checked


def test_loads_into_lds_have_their_wait_states(kernels):
    """A load into LDS is assembly text: one wait state behind the write of m0, five behind a vector operation's of a scalar
    register that the load reads.  The text has them, whatever the compiler puts in front of it."""
    checked = 0
    for name, lines in kernels.items():
        for text in _texts(lines):
            for i, line in enumerate(text):
                if not line.startswith("buffer_load"):
                    continue
                checked += 1
                states = [(int(t.split()[1]) + 1 if t.startswith("s_nop") else 1) for t in text[:i]]
                assert text[0].startswith("s_mov_b32 m0") and sum(states) >= 5 and sum(states[1:]) >= 1, (name, text)
    assert checked


def test_text_that_writes_m0_says_so():
    with open(next(s for s in B.SOURCES if os.path.basename(s) == "rows.hip")) as f:
        texts = re.findall(r"\basm\b.*?;\n", f.read(), re.S)
    wrote = [t for t in texts if re.search(r"s_mov_b32 m0", t)]
    assert wrote and all(re.search(r':\s*"memory", "m0"\)', t) for t in wrote)
