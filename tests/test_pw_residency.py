"""The choice of a pointwise MXFP4 layer's kernel on 16-bit input counts the workgroups that LDS lets run, on the host: many rows with long reductions."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
ROWS, CODES = 76, 78


@pytest.fixture
def choices(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path / "choose_pw_lds"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    str(ROOT / "include"), str(ROOT / "tests" / "host" / "choose_pw_lds.cpp"), "-o", str(exe)], check=True, capture_output=True)

    def run(shapes):
        out = subprocess.run([str(exe)], input="".join("%d %d %d\n" % s for s in shapes), capture_output=True, text=True, check=True, env={"ASAN_OPTIONS": "detect_leaks=0"}).stdout
        return dict(zip(shapes, (tuple(map(int, line.split())) for line in out.splitlines())))
    return run


# us on (rows, cin, cout): rows quantised in LDS, and a quantisation of its own with the product on its codes
MEASURED = {(12544, 4096, 4096): (252, 150), (20000, 4096, 4096): (378, 226), (32768, 4096, 4096): (544, 347), (65536, 4096, 1024): (316, 250), (20000, 4096, 8192): (703, 362),
            (32768, 8192, 1024): (343, 234), (20000, 2048, 8192): (339, 227), (20000, 2048, 2048): (100, 76), (32768, 2048, 2048): (144, 128), (65536, 2048, 2048): (291, 241),
            (32768, 1024, 16384): (985, 420), (50176, 2048, 64): (44, 63), (50176, 2048, 256): (57, 74), (401408, 384, 96): (77, 99), (50176, 512, 256): (22, 31)}


def test_the_faster_of_both(choices):
    got = choices(list(MEASURED))
    for shape, (lds, codes) in MEASURED.items():
        assert got[shape][0] == (ROWS if lds < codes else CODES), shape


def test_four_waves_where_four_workgroups_fit(choices):
    shapes = [(rows, cin, cout) for rows in (100, 12544, 32767, 32768, 65536, 401408) for cin in (257, 384, 1024, 1536, 2048, 4096, 8192) for cout in (8, 96, 1024, 4096, 8192)]
    for shape, (_, waves, resident) in choices(shapes).items():
        assert waves == (4 if shape[0] >= 32768 and resident >= 4 else 8), shape
    assert all(waves == 4 for _, waves, _ in choices([(rows, cin, 96) for rows in (1, 100000) for cin in (8, 96, 256)]).values())
