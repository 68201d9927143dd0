"""Assembly in the kernels writes only registers that the compiler gave it (read from the sources)."""
import glob
import os
import re

import pytest

from paper_1905_10308_amd.build import CSRC

FIXED = re.compile(r"^(m0|vcc\w*|exec\w*|flat_scratch\w*|scc|[sva]\d+|[sva]\[)")


def statements(text):
    """The templates of a source's assembly statements, adjacent literals joined."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(\s*((?:\"(?:[^\"\\]|\\.)*\"\s*)+)", text):
        yield "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))


def written(template):
    """The first operands of a template's instructions: what most of them write."""
    for line in re.split(r"\\n|;", template):
        words = line.replace("\\t", " ").split(None, 1)
        if len(words) == 2:
            yield words[1].split(",")[0].strip()


def test_the_reader():
    assert list(written(r"s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2")) == ["m0", "0", "%1"]
    assert list(statements('asm volatile("a %0, 1\\n\\t"\n  "b %1" : : "s"(x));  asm("" : "+v"(y));')) == [r"a %0, 1\n\tb %1", ""]
    assert FIXED.match("m0") and FIXED.match("v[2:3]") and not FIXED.match("%0") and not FIXED.match("0")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))), ids=os.path.basename)
def test_no_register_of_its_own_choice(path):
    with open(path) as f:
        for template in statements(f.read()):
            fixed = [w for w in written(template) if FIXED.match(w)]
            assert not fixed, f"{template!r} writes {fixed} behind the compiler's back"
