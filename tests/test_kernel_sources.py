"""Inline assembly of the kernels: what the compiler has to know of it stands in its constraints."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2309_06626_amd", "csrc")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        for found in re.finditer(r"\basm\s*(?:volatile)?\s*\(((?:\"(?:\\.|[^\"\\])*\"|[^\";])*)\)\s*;", open(path).read()):
            template = re.match(r"\s*((?:\"(?:\\.|[^\"\\])*\"\s*)+)", found.group(1))
            yield os.path.basename(path), template.group(1), found.group(1)[template.end():]


def test_the_statements_are_found():
    assert sum("global_load_lds" in text for _, text, _ in statements()) >= 1
    assert len(list(statements())) >= 10


def test_m0_is_named():
    """A register that a statement uses without naming it may hold something of the compiler's: m0 is the base of transfers into LDS."""
    for name, text, operands in statements():
        if re.search(r"\bm0\b", text) or re.search(r"\b(global|buffer)_load_(lds|dword\w* .*\blds\b)", text):
            assert '"{m0}"' in operands or '"m0"' in operands, (name, text)
