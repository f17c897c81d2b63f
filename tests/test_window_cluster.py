"""How many CTAs share a single token's keys: the rule itself, compiled for the host. CPU only."""
import ctypes
import shutil
import subprocess

import pytest

from paper_2609_10018_gb300 import build


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("window_cluster")
    (d / "rule.cpp").write_text('#include "window_cluster.h"\nextern "C" int rule(long long u, long long k, int s, int m) '
                                '{ return elasto::single_token_cluster(u, k, s, m); }\n')
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC, str(d / "rule.cpp"), "-o", str(d / "rule.so")], check=True)
    f = ctypes.CDLL(str(d / "rule.so")).rule
    f.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return f


SIZES = [(u, k) for u in (1, 2, 8, 19, 38, 76, 152, 304, 608, 1216, 1 << 24) for k in (1, 128, 255, 256, 1000, 4096, 9000, 40000, 1 << 30)]


@pytest.mark.parametrize("sms", [16, 76, 148, 152])
def test_no_more_than_the_device_runs(rule, sms):
    for u, k in SIZES:
        assert rule(u, k, sms, 8) == min(rule(u, k, sms, 16), 8), (u, k)
    assert any(rule(u, k, sms, 16) == 16 for u, k in SIZES)


def test_every_cta_has_keys(rule):
    for u, k in SIZES:
        n = rule(u, k, 152, 16)
        assert n in (1, 2, 4, 8, 16) and (n == 1 or k >= 128 * n), (u, k)
