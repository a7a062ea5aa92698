"""What the library asks of the CUDA runtime once and keeps is never a failure: no
static is initialised from a call that may fail."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_static_is_initialised_from_a_query():
    files = glob.glob(os.path.join(ROOT, "paper_2608_02123_gb300", "csrc", "*.cu*"))
    assert len(files) > 5
    for path in files:
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        # a static with an initialiser that is a lambda's or a call's result
        for m in re.finditer(r"\bstatic\s+(?!constexpr|__device__)[\w:<>\s*&]+=\s*", text):
            value = text[m.end():m.end() + 400].split("\n}", 1)[0]
            assert not re.match(r"\[|cuda\w+\s*\(", value), (path, m.group(0))
