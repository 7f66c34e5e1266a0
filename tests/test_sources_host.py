"""Host checks of the kernel sources' text."""
import glob
import os
import re

from tests.small_plan import ROOT


def test_no_specifier_is_written_twice():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2605_19269_amd", "csrc", "*"))):
        for number, line in enumerate(open(path), 1):
            assert not re.search(r"\b(static|inline|const|constexpr|extern|__device__|__forceinline__)\s+\1\b", line.split("//")[0]), "%s:%d" % (path, number)
