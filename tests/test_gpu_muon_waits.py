"""The limit of the waits of orthogonalised momentum's products: it bounds what a wait waits for (a copy, a tile), not a launch."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
SIDE, LIMIT_NS = 8192, 1000000


@pytest.fixture(scope="module")
def short(tmp_path_factory):
    """The library, its products' waits with a limit of a millisecond instead of a second."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    others = [os.path.join(darb_build.BUILD, os.path.splitext(s)[0] + ".o") for s in darb_build.SOURCES if s != "muon.cu"]
    darb_build.build(force=not all(os.path.exists(o) for o in others))
    at = tmp_path_factory.mktemp("waits")
    obj, out = str(at / "muon.o"), str(at / "libshort.so")
    subprocess.run([darb_build.nvcc(), "-c", os.path.join(darb_build.CSRC, "muon.cu"), "-o", obj, "-O3", "-std=c++17", *darb_build.ARCH,
                    "-Xcompiler", "-fPIC,-fvisibility=hidden", "-I", darb_build.INCLUDE, "-I", darb_build.CSRC, "-DDARB_BUILDING_LIBRARY",
                    f"-DDARB_WAIT_LIMIT_NS={LIMIT_NS}"], check=True)
    subprocess.run([darb_build.nvcc(), "-shared", obj, *others, "-o", out, *darb_build.ARCH, "-Xcompiler", "-fPIC", "-ldl"], check=True)
    lib = ctypes.CDLL(out)
    for name in ("create", "step", "sync_status", "destroy"):
        getattr(lib, "darb_muon_" + name).argtypes = getattr(darb.lib(), "darb_muon_" + name).argtypes
    return lib


def test_a_launch_longer_than_the_limit(short):
    """Products of 8192 x 8192 by 8192 x 8192, three for each, take over 2 ms a launch at the tensor cores' 1.95 PFLOP/s
    at most (6 * 8192^3 / 1.95e15 = 1.7 ms), and 0.15 ms a tile: no wait gives up, and the step is the ordinary one's."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    p, m, g = (torch.randn(SIDE, SIDE, generator=gen, device="cuda") * s for s in (0.1, 1e-3, 1e-3))
    want_p, want_m = p.clone(), m.clone()
    with darb.darb_muon_create([want_p], [want_m]) as plan:
        darb.darb_muon_step(plan, [g], 0.05)
        darb.darb_muon_sync_status(plan)
    side, pointers = (ctypes.c_int64 * 1)(SIDE), [(ctypes.c_void_p * 1)(t.data_ptr()) for t in (p, m, g)]
    plan, stream = ctypes.c_void_p(), torch.cuda.current_stream().cuda_stream
    assert short.darb_muon_create(1, side, side, pointers[0], pointers[1], None, darb.F32, ctypes.byref(plan), stream) == darb.OK
    assert short.darb_muon_step(plan, pointers[2], None, 0.05, 0.95, 0.01, 1e-7, 1, stream) == darb.OK
    status = short.darb_muon_sync_status(plan, stream)
    assert short.darb_muon_destroy(plan) == darb.OK
    assert torch.equal(p, want_p) and torch.equal(m, want_m)
    assert status == darb.OK
