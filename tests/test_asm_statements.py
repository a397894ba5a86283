"""What inline assembly of the kernels has to say of itself (no GPU needed)."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2408_01391_amd" / "csrc"


def statements(text):
    """(instructions, clobbers) of every asm statement."""
    for at in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        depth, i, quoted = 1, at.end(), False
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        parts, depth, quoted = [""], 0, False
        for c in text[at.end():i - 1]:
            if c == '"':
                quoted = not quoted
            depth += 0 if quoted else (c in "([") - (c in ")]")
            if c == ":" and not quoted and depth == 0:
                parts.append("")
            else:
                parts[-1] += c
        yield "".join(re.findall(r'"([^"]*)"', parts[0])), re.findall(r'"([^"]*)"', parts[3]) if len(parts) > 3 else []


def test_statements_are_found():
    text = 'asm volatile("s_mov_b32 m0, %0\\n\\t" "x" ::"s"(f(a[1 ? 2 : 3])) : "memory", "m0"); asm("");'
    assert list(statements(text)) == [("s_mov_b32 m0, %0\\n\\tx", ["memory", "m0"]), ("", [])]


@pytest.mark.parametrize("path", sorted(p.name for p in CSRC.iterdir() if p.suffix in (".h", ".hip")))
def test_m0_is_named_where_it_is_written(path):
    for text, clobbers in statements((CSRC / path).read_text()):
        if re.search(r"\bs_\w+ m0\b", text):
            assert "m0" in clobbers, text
