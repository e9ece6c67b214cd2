"""What the kernel sources must not do, checked without a GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_00596_amd", "csrc")


def _asm(text):
    """The instruction text of every asm statement."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        end, depth = m.end(), 1
        while depth:
            depth += {"(": 1, ")": -1}.get(text[end], 0)
            end += 1
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text[m.end():end].split(":")[0]))


def test_vector_instructions_in_asm_wait_for_matrix_results():
    """The compiler keeps a distance between a matrix instruction and the vector instruction that reads its result, but not where that one is an asm
    statement.  A file that has such statements waits for the results by itself (results_ready, which holds the waits), or has no matrix results
    there; so far one file does."""
    found = set()
    for path in glob.glob(os.path.join(CSRC, "*")):
        if os.path.isfile(path) and path.endswith((".hip", ".h", ".cpp")):
            text = re.sub(r"//[^\n]*", "", open(path).read())
            if any(re.search(r"\bv_\w+", a) for a in _asm(text)):
                found.add(os.path.basename(path))
    assert found == {"small_channel_rows_kernel.hip"}, found
    text = open(os.path.join(CSRC, "small_channel_rows_kernel.hip")).read()
    assert re.search(r"void results_ready\(.*\n\{\n\s*asm volatile\(\"s_nop 15\\n\\ts_nop 7\"", text) and text.count("results_ready(") >= 2
