"""Loads that are defined while another kernel writes.

These kernels are launched before the one ahead of them in the stream has ended, and what they read it may have
written: they wait for it, but a load through the read-only path (``__ldg``, ``ld.global.nc``) is defined only for data
that nothing writes from the kernel's start on, and a compiler may move it to before the wait.  A race of this kind is
not shown by running it, so the sources are looked at."""
import os
import re

import pytest

from paper_1911_08020_gb300.build import CSRC


@pytest.mark.parametrize("name", ["adamw.cu", "layer_norm.cu", "logprobs.cu", "muon.cu", "policy.cu", "scan.cu", "tokens.cuh"])
def test_no_read_only_loads(name):
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    assert "pdl_wait_previous" in code or name.endswith(".cuh")
    assert not re.search(r"__ldg\b|\.nc\b|__restrict__", code)
