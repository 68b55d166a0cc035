"""Which kernel a pointwise layer on FP8 blocks takes, on the host: measured layers where they belong, and nothing that its kernel does not take."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
TILE64, TILE128, TILE256, FEW32, FEW64, FEW16, ROWS, ROWS128, CODES = range(80, 89)


def _choices(tmp_path, shapes):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path / "choose_f8"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    str(ROOT / "include"), str(ROOT / "tests" / "host" / "choose_f8.cpp"), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], input="".join("%d %d %d\n" % s for s in shapes), capture_output=True, text=True, check=True, env={"ASAN_OPTIONS": "detect_leaks=0"}).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_measured_layers(tmp_path):
    """(rows, cin, cout): the kernels on codes and on 16-bit input that took the least time of those measured, or within 8 %."""
    want = {(1, 2048, 1000): (FEW32, FEW16), (16, 1024, 4096): (FEW32, FEW16), (16, 8192, 8192): (FEW32, CODES), (32, 4096, 4096): (FEW32, CODES), (100, 4096, 4096): (TILE64, CODES),
            (1531, 1000, 777): (TILE64, ROWS), (200704, 64, 256): (TILE128, ROWS128), (401408, 96, 384): (TILE128, ROWS128), (401408, 64, 64): (TILE64, ROWS128),
            (50176, 256, 512): (TILE128, ROWS), (12544, 1024, 256): (TILE128, ROWS), (12544, 8192, 1024): (TILE256, CODES), (2048, 4096, 4096): (TILE128, CODES),
            (20000, 2048, 2048): (TILE128, CODES), (8192, 8192, 8192): (TILE256, CODES)}
    assert {shape: choice[:2] for shape, choice in zip(want, _choices(tmp_path, want))} == want


def test_everything_chosen_fits(tmp_path):
    shapes = [(rows, cin, cout) for rows in (1, 2, 31, 32, 33, 64, 65, 1000, 32768, 32769, 2 ** 31 - 1) for cin in (1, 63, 64, 96, 128, 129, 1000, 8192, 65536, 2 ** 20, 2 ** 22)
              for cout in (1, 33, 255, 256, 1024, 8192, 65536) if cin * cout < 2 ** 31]
    for shape, (codes, wide, fits, splits) in zip(shapes, _choices(tmp_path, shapes)):
        assert fits and TILE64 <= codes <= FEW64 and FEW16 <= wide <= CODES and splits >= 1, shape
        assert wide != FEW16 or shape[0] <= 32, shape
