"""The host side of dropout, log probabilities and cross entropy under a check for undefined arithmetic (no GPU: the launches go to
tests/fake_hip.cpp): shifts and sums of every kind of format, dense and strided, small, long and many rows."""
import os
import subprocess

import pytest

from test_launch_limits import ROOT, _run

CALLS = """
import os
host = C.CDLL(os.environ["HEAD_HOST_LIB"])
for name in ("adapt_dropout", "adapt_log_probs", "adapt_cross_entropy"):
    getattr(host, name).argtypes = getattr(lib, name).argtypes
h = context()
F, R = b.Fmt, b.Rng(1, 1, 1)
formats = [F(wl, fl) for wl in (2, 8, 9, 16, 17, 32) for fl in (0, 4, 31)]
calls = 0
for f in [F(0, 0), F(0, 7)] + formats:
    for rows, classes, ld in ((0, 5, 5), (1, 1, 1), (9, 256, 300), (9, 257, 257), (3, 200003, 1 << 20), (4000, 50000, 50000), ((1 << 31) - 1, 512, 512), (1, 1 << 30, 1 << 40)):
        assert host.adapt_log_probs(h, at, f, rows, classes, ld, 2 * at, 3 * at, 4 * at, 5 * at, min(32, classes), 6 * at, 7 * at) == 0
        for fg in (F(2, 0), F(8, 7), F(16, 31), F(32, 0)):
            assert host.adapt_cross_entropy(h, at, f, rows, classes, ld, 2 * at, 3 * at, fg, R, 9 * at, ld, 7 * at) == 0
        calls += 5
for fx in formats:
    for fo in formats:
        for p in (0.0, 0.3, 65535 / 65536):
            for res, fres in ((None, fx), (at, F(8, 0)), (at, F(32, 31))):
                want = -2 if fo.fl - fx.fl > 15 or (res and fres.fl > fo.fl) else 0
                assert host.adapt_dropout(h, 2 * at, fx, 1 << 40, p, fo, R, res, fres, 3 * at + (1 << 45)) == want
                calls += 1
print(calls, len(fake.fake_launched().split()))
"""


def test_the_host_arithmetic_is_defined(tmp_path, monkeypatch):
    lib, csrc = str(tmp_path / "libhead_host.so"), os.path.join(ROOT, "paper_2107_13490_amd", "csrc")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wno-unused-function",
                    "-fuse-cuid=none", "-Wl,--defsym=__hip_fatbin=0,--allow-multiple-definition",      # there is no device code
                    "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fsanitize-trap=undefined",
                    "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "logits.hip"), os.path.join(csrc, "dropout.hip"), "-o", lib], check=True)
    monkeypatch.setenv("HEAD_HOST_LIB", lib)
    calls, launches = (int(v) for v in _run(CALLS, tmp_path).split())
    assert calls > 2000 and launches > 2000
