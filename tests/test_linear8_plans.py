"""Which tiles the kernel of 8-bit layers for many tokens takes for the sizes that it is tested at: every kind of tile, workgroups with one tile and with several,
products shorter than the copies that are on their way and longer ones.  On the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (rows, channels, K): (32 channels of a tile, slabs of 16 rows of a wavefront at most, steps of 64 k, tiles of a workgroup at most)
SIZES = {
    (65, 16388, 80): (8, 1, 2, 1),
    (65, 80004, 64): (8, 2, 1, 2),
    (257, 40004, 144): (8, 2, 3, 2),
    (300, 40000, 208): (8, 2, 4, 2),
    (300, 40004, 1040): (8, 2, 17, 2),
    (1000, 16388, 336): (8, 3, 6, 2),
    (515, 13824, 192): (8, 3, 3, 1),
    (1500, 16384, 64): (8, 3, 1, 2),
    (2309, 13824, 5120): (8, 3, 80, 3),
    (3000, 8196, 512): (8, 4, 8, 2),
    (2309, 5120, 1040): (8, 4, 17, 1),
    (2100, 28676, 80): (8, 4, 2, 4),
    (65, 8196, 64): (4, 1, 1, 1),
    (100, 16388, 128): (4, 2, 2, 1),
    (257, 8200, 448): (4, 2, 7, 1),
    (130, 80004, 144): (4, 3, 3, 3),
    (257, 13820, 192): (4, 3, 3, 1),
    (700, 8192, 1024): (4, 3, 16, 1),
    (700, 9000, 320): (4, 4, 5, 1),
    (130, 516, 272): (2, 1, 5, 1),
    (65, 8200, 1040): (2, 2, 17, 1),
    (130, 13828, 96): (2, 3, 2, 1),
    (130, 13824, 1040): (2, 3, 17, 1),
    (1500, 2052, 256): (2, 4, 4, 1),
    (1500, 2056, 832): (2, 4, 13, 1),
}


def test_sizes_take_the_tiles_that_they_are_here_for(tmp_path):
    exe = str(tmp_path / "plans")
    build = subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "paper_2305_10727_amd", "csrc"),
                            os.path.join(ROOT, "tests", "linear8_plans.cpp"), "-o", exe], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([exe], input="".join("%d %d %d\n" % s for s in SIZES), capture_output=True, text=True, timeout=60)
    got = dict(zip(SIZES, (tuple(map(int, line.split())) for line in run.stdout.splitlines())))
    assert got == SIZES
    # every kind of tile; of the ones of 256 channels those with several slabs also by workgroups with several tiles
    assert {t[:2] for t in got.values()} == {(tn, nx) for tn in (8, 4, 2) for nx in (1, 2, 3, 4)}
    assert {t[:2] for t in got.values() if t[3] > 1} >= {(8, 2), (8, 3), (8, 4), (4, 3)}
