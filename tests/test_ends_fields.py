"""What the structs of the operators at the model's two ends hold is read: a kernel's arguments by a
kernel or a launch, a plan's parts by the checks or the launches."""
import os
import re

import pytest

from test_dependent_kernels import CSRC


@pytest.mark.parametrize("name", ["hcw_embed.cu", "hcw_clip.cu", "hcw_q4.cu", "hcw_logits.cu"])
def test_every_field_is_read(name):
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, name)).read(), flags=re.S)
    seen = 0
    for m in re.finditer(r"struct (\w+) \{\n(.*?)\n\};", text, flags=re.S):
        if "(" in m.group(2):     # has functions
            continue
        # a kernel's arguments are `a` there
        var = "a" if m.group(1).endswith("Args") else r"\w+(?:\[\w+\])?"
        for line in m.group(2).split(";"):
            for field in re.findall(r"[\s*](\w+)(?:\[[^\]]*\])?(?=\s*(?:,|$))", line):
                seen += 1
                assert re.search(r"\b%s\.%s\b(?!(?:\[\w+\])? = )" % (var, field), text), (m.group(1), field)
    assert seen > 5
