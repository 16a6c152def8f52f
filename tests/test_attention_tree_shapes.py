"""Which kernel a tree's attention takes, on the host: columns of 16 that share the keys, or with keys dealt out, as measured on either side."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (padded head, pairs of sequence and key head, columns): the kernel for many columns
TREES = {
    (128, 8, 192): 0, (128, 8, 193): 1, (128, 16, 192): 0, (128, 16, 208): 1, (128, 32, 256): 1, (128, 63, 193): 1, (128, 64, 256): 0, (128, 128, 256): 0, (128, 128, 257): 1,
    (64, 8, 192): 0, (64, 15, 193): 1, (64, 16, 256): 0, (64, 32, 256): 0, (64, 128, 257): 1, (256, 16, 32): 0, (256, 128, 33): 1, (128, 1, 17): 0, (128, 512, 16): 0,
}


def test_trees_take_the_faster_kernel(tmp_path):
    exe = str(tmp_path / "shapes")
    build = subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "paper_2305_10727_amd", "csrc"),
                            os.path.join(ROOT, "tests", "attend_shapes.cpp"), "-o", exe], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([exe], input="".join("%d %d %d\n" % t for t in TREES), capture_output=True, text=True, timeout=60)
    assert dict(zip(TREES, map(int, run.stdout.split()))) == TREES
