"""The walk that the kernels of token log probabilities take where more elements reach
their bound than a list holds, on the CPU with a thread that is late whenever it reads
the list's counter: all threads come to the same steps, none waits for ever, and the
list ends with the best."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("walk") / "driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-pthread",
                        "-I", os.path.join(ROOT, "paper_2607_05804_amd", "csrc"),
                        os.path.join(ROOT, "tests", "candidate_walk_driver.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


# packs, elements of a pack, least room, threads, capacity, k: steps that the room limits
# (the row kernel) and steps of all threads (the join), with and without a cut
@pytest.mark.parametrize("sizes", [(200, 8, 32, 8, 64, 5), (333, 4, 16, 8, 40, 12), (7, 8, 32, 8, 64, 5),
                                   (1, 8, 32, 8, 64, 5), (0, 8, 32, 8, 64, 5), (300, 1, 8, 8, 28, 4),
                                   (8, 1, 8, 8, 28, 4)])
@pytest.mark.parametrize("late", [0, 5])
def test_a_late_thread_takes_the_same_steps(sizes, late, driver):
    r = subprocess.run([driver, *map(str, sizes), str(late)], capture_output=True, text=True, timeout=120)
    assert r.stdout == "ok\n", r.stdout + r.stderr
