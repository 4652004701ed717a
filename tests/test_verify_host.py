"""Checks of the verifying pass's sources and launches that need no GPU."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_assembly_that_writes_m0_says_so():
    """The compiler keeps values of its own in m0 (indexes, messages) across statements that do not name it."""
    found = 0
    for name in glob.glob(os.path.join(ROOT, "paper_2503_05330_amd", "csrc", "*")):
        for body in re.findall(r"\basm\b[^;]*?\((.*?)\);", open(name).read(), re.S):
            writes = re.search(r"[sv]_\w+\s+m0\b", body)
            if writes:
                found += 1
                assert re.search(r'"m0"[^:]*$', body), (name, body)
    assert found == 4
