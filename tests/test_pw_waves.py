"""Waves of the few-row MXFP4 kernel, on the host: elements are counted in 64 bits, whatever the layer."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


def test_waves_of_small_and_large_layers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path / "choose_pw_waves"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    str(ROOT / "include"), str(ROOT / "tests" / "host" / "choose_pw_waves.cpp"), "-o", str(exe)], check=True, capture_output=True)
    # scale words (256 channels each) and elements decide; 401408 x 8192 and more pass 2^31 elements
    want = {(1, 256, 8): 4, (1, 1024, 8): 4, (1, 1025, 8): 8, (1, 2048, 1000): 8, (1, 2049, 8): 16, (8, 1024, 64): 4, (9, 1024, 64): 8, (16, 1024, 64): 8, (17, 1024, 64): 16,
            (32, 256, 64): 4, (32, 8192, 64): 16, (401408, 8192, 256): 16, (401408, 5352, 8): 16, (2 ** 31 - 1, 3, 8): 16, (2 ** 31 - 1, 2 ** 24, 1): 16}
    out = subprocess.run([str(exe)], input="".join("%d %d %d\n" % s for s in want), capture_output=True, text=True, check=True, env={"ASAN_OPTIONS": "detect_leaks=0"}).stdout
    assert dict(zip(want, map(int, out.split()))) == want
