"""How the kernels read what the kernel before them may still be writing: they are launched while it runs, and wait for it inside, so no
load of theirs may promise that its data stays as it is for the kernel's whole life."""
import glob
import os
import re

import pytest

import paper_2607_19456_b200 as moa

CSRC = os.path.join(os.path.dirname(moa.__file__), "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_no_load_through_the_read_only_path(path):
    with open(path) as f:
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    assert not re.findall(r"__ldg\s*\(|\bld\.global(?:\.\w+)*\.nc\b|__restrict__", text)
