"""Kernels that may start before the kernel in front of them has finished see memory only behind
pdl_wait: it is what makes visible the writes of the kernel in front, and of what lies before that
one.  So every thread waits, whatever the call, and the operators at the model's two ends name no
tensor before they do."""
import glob
import os
import re

import pytest

from test_dependent_kernels import CSRC, kernels

ENDS = ("hcw_embed.cu", "hcw_clip.cu", "hcw_q4.cu", "hcw_logits.cu")


def source(name):
    return open(os.path.join(CSRC, name)).read()


def test_the_wait_is_under_no_condition():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        for name, body in kernels(open(path).read()):
            if "pdl_wait()" not in body:
                continue
            seen += 1
            assert not re.search(r"(\bif\s*\([^;{}]*\)|\belse)\s*pdl_wait\(\)", body), name
    assert seen > 30


def pointers(text):
    """Names of the pointers in the argument structs of a source."""
    found = set()
    for m in re.finditer(r"struct \w+(?:Args|Tensor) \{(.*?)\n\};", text, flags=re.S):
        found |= set(re.findall(r"\*\s*(\w+)(?:\[\d+\])?;", m.group(1)))
    return found


@pytest.mark.parametrize("name", ENDS)
def test_no_tensor_is_named_before_the_wait(name):
    text = source(name)
    members = pointers(text)
    seen = 0
    for kernel, body in kernels(text):
        at = body.index("{")
        args = set(re.findall(r"\*\s*(?:const\s+)?(\w+)\s*[,)]", body[body.index(kernel):at]))
        # up to the first wait that is a statement of its own
        wait = re.search(r"[;{}]\s*pdl_wait\(\)", body[at:])
        assert wait, kernel
        before = body[at:at + wait.start()]
        seen += 1
        used = {v for v in args if re.search(r"\b%s\b" % v, before)}
        used |= {v for v in members if re.search(r"\ba\s*\.\s*%s\b" % v, before)}
        assert not used, (kernel, sorted(used))
        assert members or args
    assert seen
