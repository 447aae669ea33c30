"""The attention's parts and tiles on the CPU: attend_tiles_driver.cpp walks them as the kernels do,
with the host compiler's checks of bounds and overflow."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2608_20375_amd", "csrc")


def test_parts_tiles_and_buffers(tmp_path):
    exe = str(tmp_path / "tiles")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-D_GLIBCXX_ASSERTIONS", "-I", CSRC, "-o", exe,
                    os.path.join(HERE, "attend_tiles_driver.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_the_kernels_use_this_arithmetic():
    """Every tile buffer's size is an extent, every part and tile the shared functions'."""
    text = open(os.path.join(CSRC, "k_attend.hip")).read()
    sizes = [l for l in text.splitlines() if "= buffer(" in l]
    assert sizes and all("extent(" in l for l in sizes), sizes
    assert text.count("part_of(") == 2 and "spot_of(" in text and "cut_tiles(" in text
