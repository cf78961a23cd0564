"""Inline assembly of the kernels says what it changes."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def statements():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2106_06601_amd", "csrc", "*.h*"))):
        text = open(path).read()
        for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", text, re.S):
            yield os.path.basename(path), m.group(1)


def test_special_registers_that_are_written_are_clobbered():
    found = 0
    for name, body in statements():
        code, _, lists = body.partition(":")
        clobbers = lists.split(":")[-1]
        for register in ("m0", "vcc", "exec", "scc"):
            if re.search(r"\b[sv]_\w+\s+%s\b" % register, code):
                found += 1
                assert '"%s"' % register in clobbers, (name, register, body)
    assert found
