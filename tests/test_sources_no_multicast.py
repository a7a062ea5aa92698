"""The library is one shared object, loaded by every rank of a run on several
GPUs: none of its TMA copies multicasts into the CTAs of a cluster."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_copy_multicasts():
    files = glob.glob(os.path.join(ROOT, "paper_2608_02123_gb300", "csrc", "*.cu*"))
    assert len(files) > 5
    for path in files:
        with open(path) as f:
            text = f.read()
        # an instruction's text may be split over adjacent literals
        text = re.sub(r'"\s*"', "", text)
        for copy in re.findall(r"cp\.async\.bulk[\w.:]*", text):
            assert "multicast" not in copy, (path, copy)
