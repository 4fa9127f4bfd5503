"""The library holds no kernel that no call reaches."""

import re
import shutil
import subprocess

import pytest

from tests.helpers import ensure_built


def test_lists_of_more_than_64_have_wide_workgroups_alone():
    """Rows whose lists hold up to 256 are taken by 512 threads; only their parts by 256."""
    from paper_2608_28726_amd.build import LIB
    ensure_built()
    if shutil.which("nm") is None:
        pytest.skip("nm is not installed")
    names = subprocess.run(["nm", "-C", LIB], capture_output=True, text=True, check=True).stdout
    found = set(re.findall(r"(top_kernel|beam_rows_kernel|top_parts_kernel)<[\w ]+, (\d+), (\d+)>", names))
    blocks = {(kernel, kept): {b for x, b, y in found if (x, y) == (kernel, kept)} for kernel, _, kept in found}
    assert blocks == {("top_kernel", "64"): {"256", "512"}, ("top_kernel", "256"): {"512"},
                      ("beam_rows_kernel", "64"): {"256", "512"}, ("beam_rows_kernel", "256"): {"512"},
                      ("top_parts_kernel", "64"): {"256"}, ("top_parts_kernel", "256"): {"256"}}
