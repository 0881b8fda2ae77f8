"""Edges of the training operators' host side (CPU: nothing here is launched)."""
import os
import subprocess
import sys

import pytest

from paper_2401_13660_gb300 import mbscan as mb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 40   # an aligned, never-dereferenced stand-in for a device address


def _at(i):
    return FAKE + (i << 34)


@pytest.mark.parametrize("n, vocab, width", [(0, 256, 64), (10, 0, 64), (10, 256, 0), (0, 256, 0), (10, 0, 0), (0, 0, 0)])
def test_embed_backward_workspace_of_nothing(n, vocab, width):
    # in a process of its own: what divides by a size ends it
    code = f"from paper_2401_13660_gb300 import mbscan as mb; print(mb.mb_embed_backward_workspace_size({n}, {vocab}, {width}))"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0 and int(r.stdout) >= 256, (r.returncode, r.stderr)
    need, lib = int(r.stdout), mb.load_library()
    call = lambda wb: lib.mb_embed_backward(_at(0), 0, _at(1), 0, 1.0, 1, _at(2), n, vocab, width, _at(3), wb, None)
    assert call(need) == mb.MB_OK   # nothing to add, so nothing is launched
