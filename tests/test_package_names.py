"""Every function of the C ABI that the binding has is a name of the package too, and every name of the package is there."""
import os
import re

import paper_2401_13660_gb300 as package
from paper_2401_13660_gb300 import mbscan as mb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_names():
    with open(os.path.join(ROOT, "include", "mbscan.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = set(re.findall(r"\b(mb_\w+)\s*\(", text))
    assert {"mb_conv1d", "mb_matmul_q8", "mb_sample"} <= declared
    lib = mb.load_library()
    assert all(hasattr(lib, name) for name in declared)
    missing = {name for name in declared if hasattr(mb, name)} - set(package.__all__)
    assert not missing, missing
    assert all(getattr(package, name) is getattr(mb, name) for name in package.__all__)
