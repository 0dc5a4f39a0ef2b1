"""The kernels' sources are linked into one library: a function of a namespace has one definition."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_02620_amd", "csrc")


def test_a_device_function_is_defined_in_one_source():
    seen = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        # at the start of a line, with external linkage: not static, no kernel (those have their arguments' types in their names)
        for m in re.finditer(r"^(?!static)(?:[\w:<>*&, ]*__(?:device|host)__[^\n(]*?)(\w+)\(", text, re.M):
            if "static" not in m.group(0):
                seen.setdefault(m.group(1), set()).add(os.path.basename(path))
    assert len(seen) > 20, "the pattern finds the functions"
    assert {name: files for name, files in seen.items() if len(files) > 1} == {}
