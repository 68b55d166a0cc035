"""How the output of a pointwise MXFP4 layer with rows in LDS leaves, on the host: past the caches where that was measured to be faster."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent

# (rows, cin, cout, residual): us by the caches and past them
MEASURED = {(200704, 64, 64, 1): (22.1, 16.4), (401408, 64, 64, 1): (38.3, 28.2), (12544, 64, 256, 1): (7.8, 6.0), (25088, 64, 256, 1): (12.0, 8.8), (50176, 64, 256, 1): (15.7, 14.3),
            (100352, 64, 256, 1): (32.5, 24.8), (200704, 64, 256, 1): (58.0, 42.0), (401408, 64, 256, 1): (127.8, 90.2), (50176, 96, 384, 1): (22.7, 22.0), (200704, 96, 384, 1): (104.1, 61.1),
            (50176, 128, 512, 1): (26.8, 25.4), (12544, 256, 1024, 1): (17.3, 15.7), (50176, 256, 512, 1): (31.0, 29.2), (401408, 96, 384, 0): (126, 66), (200704, 96, 384, 0): (46, 52)}


def test_the_faster_way(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path / "choose_pw_stores"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    str(ROOT / "include"), str(ROOT / "tests" / "host" / "choose_pw_stores.cpp"), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], input="".join("%d %d %d %d\n" % s for s in MEASURED), capture_output=True, text=True, check=True, env={"ASAN_OPTIONS": "detect_leaks=0"}).stdout
    assert [int(line) for line in out.split()] == [int(past < kept) for kept, past in MEASURED.values()]
