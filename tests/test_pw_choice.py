"""Which kernel a pointwise MXFP4 layer takes, on the host: measured layers on the side of each line where they belong, and nothing that its kernel does not take."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
TILE64, TILE128, TILE256, FEW32, FEW64, FEW16, ROWS, ROWS128, CODES = range(70, 79)


def _choices(tmp_path, shapes):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path / "choose_pw"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    str(ROOT / "include"), str(ROOT / "tests" / "host" / "choose_pw.cpp"), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], input="".join("%d %d %d\n" % s for s in shapes), capture_output=True, text=True, check=True, env={"ASAN_OPTIONS": "detect_leaks=0"}).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_measured_layers(tmp_path):
    """(rows, cin, cout): the kernels on codes and on 16-bit input that took the least time of all that fit, within 3 %."""
    want = {(1, 2048, 1000): (FEW32, FEW16), (16, 1024, 4096): (FEW32, FEW16), (16, 8192, 8192): (FEW32, CODES), (32, 8192, 1024): (FEW32, CODES),
            (33, 8192, 8192): (FEW64, CODES), (100, 768, 2304): (FEW32, ROWS), (196, 2048, 512): (FEW32, CODES), (100, 4096, 4096): (TILE64, CODES),
            (512, 4096, 4096): (TILE64, CODES), (1024, 8192, 8192): (TILE128, CODES), (3136, 256, 1024): (TILE128, ROWS), (12544, 1024, 256): (TILE128, ROWS),
            (200704, 256, 64): (TILE64, ROWS128), (200704, 96, 384): (TILE128, ROWS128), (401408, 96, 96): (TILE128, ROWS128), (12544, 8192, 1024): (TILE256, CODES),
            (8192, 8192, 8192): (TILE256, CODES)}
    got = {shape: choice[:2] for shape, choice in zip(want, _choices(tmp_path, want))}
    assert got == want


def test_everything_chosen_fits(tmp_path):
    shapes = [(rows, cin, cout) for rows in (1, 2, 31, 32, 33, 64, 65, 1000, 32768, 32769, 2 ** 31 - 1) for cin in (1, 31, 32, 96, 256, 257, 1000, 8192, 65536, 2 ** 20)
              for cout in (1, 33, 255, 256, 1024, 8192, 65536) if cin * cout < 2 ** 31]
    for shape, (codes, wide, fits, splits) in zip(shapes, _choices(tmp_path, shapes)):
        assert fits and TILE64 <= codes <= FEW64 and FEW16 <= wide <= CODES and splits >= 1, shape
        assert wide != FEW16 or shape[0] <= 32, shape
