"""A wait of the attention kernels that runs out: the kernel returns in time, its
code is reported once to each asker, and what follows is clean."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("native") / "wait_probe.so")
    r = subprocess.run([build.nvcc(), *build.ARCH, *build.FLAGS, "-shared", "-o", so,
                        os.path.join(ROOT, "tests", "native", "wait_probe.cu")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    torch.zeros(1, device="cuda")
    L = C.CDLL(so)
    L.probe_wait.argtypes = [C.c_uint64, C.c_int, C.c_void_p]
    L.probe_told.argtypes = [C.c_void_p, C.c_void_p]
    return L


def told(L, seen):
    code = C.c_int(-1)
    assert L.probe_told(C.byref(seen), C.byref(code)) == 0
    return code.value


def test_a_wait_that_runs_out(probe):
    a, b = C.c_uint(0), C.c_uint(0)
    assert told(probe, a) == 0
    out = (C.c_ulonglong * 4)()
    limit = 1000000                                  # 1 ms
    assert probe.probe_wait(limit, 70, out) == 0     # the kernel returned and the context is usable
    assert out[3] == 3
    # the limit is looked at after 64 attempts, each of which the hardware may hold for a while
    assert limit <= out[0] < 2000 * limit and limit <= out[2] < 2000 * limit
    assert out[1] < limit                            # after the first, the same role does not wait again
    assert told(probe, a) in (70, 72) and told(probe, a) == 0
    assert told(probe, b) in (70, 72) and told(probe, b) == 0       # the other asker hears of it too, once
    assert probe.probe_wait(limit, 80, out) == 0
    assert told(probe, a) in (80, 82) and told(probe, b) in (80, 82) and told(probe, a) == 0


def test_the_context_stays_usable(probe):
    out = (C.c_ulonglong * 4)()
    assert probe.probe_wait(1000000, 90, out) == 0
    q = torch.randn(1, 128, 2, 64, device="cuda").bfloat16()
    o, lse = api.attention_forward(q, q, q)
    api.attention_error()
    api.attention_error()
    assert bool(torch.isfinite(o.float()).all())
