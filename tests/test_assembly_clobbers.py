"""Instructions written by hand in the kernels' sources: a register that they name themselves and write is among what they tell the compiler
that they change."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = sorted(p for k in ("*.hip", "*.inc", "*.h") for p in glob.glob(os.path.join(ROOT, "paper_2506_15976_amd", "csrc", k)))


def statements(text):
    """(instructions, list of what they change) of every asm statement."""
    for start in re.finditer(r"\basm\s+(?:volatile\s*)?\(", text):
        depth, at = 1, start.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        parts = re.split(r":(?=(?:[^\"]*\"[^\"]*\")*[^\"]*$)", text[start.end():at - 1])
        yield "".join(re.findall(r'"([^"]*)"', parts[0])), re.findall(r'"([^"]*)"', parts[3]) if len(parts) > 3 else []


def test_registers_that_assembly_writes_are_named():
    seen = 0
    for path in SOURCES:
        with open(path) as f:
            text = f.read()
        for code, changed in statements(text):
            seen += 1
            for line in re.split(r"\\n(?:\\t)?|;", code):
                words = line.replace(",", " ").split()
                if len(words) > 1 and re.fullmatch(r"m0|vcc|exec|scc|[sva]\d+|[sva]\[\d+:\d+\]", words[1]):
                    assert words[1] in changed, f"{os.path.basename(path)}: {line} changes {words[1]}"
    assert seen > 10
