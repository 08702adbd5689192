"""Loads that are defined while another kernel writes.

These kernels are launched before the one ahead of them in the stream has ended, and what they read it may have
written: they wait for it, but a load through the read-only path (``__ldg``, ``ld.global.nc``, what ``__restrict__``
allows) is defined only for data that nothing writes from the kernel's start on, and a compiler may move it to before
the wait.  A race of this kind is not shown by running it, so the sources are looked at."""
import os
import re

import pytest

from paper_1911_08020_gb300.build import CSRC


# Not launched that way: these begin when everything before them has ended.
PLAIN = {"assign.cu", "sequence.cu", "noalloc.cu", "baselines.cu"}
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh")) and f not in PLAIN)


def code_of(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


# Tables that the host has copied before a handle is given out, and no kernel writes.
TABLES = {"encode.cu": ["u.v[0] = __ldg(q);", "u.v[1] = __ldg(q + 1);"], "batch.cuh": ["const WorkItem *__restrict__ items"],
          "xres.cuh": ['asm volatile("ld.global.nc.v4.s32'] * 3}


@pytest.mark.parametrize("name", SOURCES)
def test_no_read_only_loads(name):
    code = code_of(name)
    for text in TABLES.get(name, ()):
        assert text in code
        code = code.replace(text, "", 1)
    assert not re.search(r"__ldg\b|\.nc\b|__restrict__", code)


@pytest.mark.parametrize("name", sorted(PLAIN))
def test_kernels_that_begin_after_all_before_them(name):
    code = code_of(name)
    assert "pdl_wait_previous" not in code and "griddepcontrol" not in code
    assert not re.search(r"launch_ex\([^;]*?stream, \w+, true", code, flags=re.S)
