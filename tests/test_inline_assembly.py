"""Inline assembly brings its own wait states: a memory access reads the scalar registers among its operands at the earliest five wait states into the block, since a vector instruction
may have written them right before it and the compiler does not look inside."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_16274_amd", "csrc")


def blocks():
    """(file, code, operands) of every block."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"\basm\s+volatile\s*\(", text):
            at, depth, k = m.end(), 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[k], 0)
                k += 1
            code = re.match(r'(\s*"(?:[^"\\]|\\.)*")+', text[at:k - 1]).group(0)
            yield os.path.basename(path), code, text[at + len(code):k - 1]


def _instructions(code):
    return [i.strip() for i in re.split(r"\\n(?:\\t)?", "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', code))) if i.strip()]


def test_wait_states_before_memory_accesses():
    seen = 0
    for name, code, operands in blocks():
        waited = 0
        for i in _instructions(code):
            if re.match(r"(global|buffer|flat|scratch)_", i):
                if not re.search(r'"(s|\{m0\})"', operands):
                    continue
                seen += 1
                assert waited >= 5, (name, code)
            nop = re.match(r"s_nop\s+(\d+)", i)
            waited += int(nop.group(1)) + 1 if nop else 1
    assert seen >= 2                                             # (the sources are read as meant)


def test_m0():
    """An access to LDS behind m0 gets it as an operand, and a block that writes m0 names it, or the compiler may keep a value there across it."""
    using = [(name, code, operands) for name, code, operands in blocks() if re.search(r"\bm0\b|_lds_", code)]
    assert len(using) >= 2
    for name, code, operands in using:
        if "_lds_" in code:
            assert '"{m0}"' in operands, (name, code)
        if re.search(r"\bs_\w+\s+m0\b", code):
            assert '"m0"' in operands.rsplit(":", 1)[1], (name, code)
