"""The short convolution's cut of a call between threads (short_conv.hpp), on
the host: no thread reads the carried state beside the ones that write it."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe = str(tmp_path_factory.mktemp("cut") / "cut")
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-O1",
                           "-fsanitize=undefined", "-fno-sanitize-recover=all", "-o", exe,
                           os.path.join(ROOT, "tests", "sanitize", "shortconv_cut.cpp")])
    return exe


def test_state_is_read_by_its_writers_alone(walk):
    r = subprocess.run([walk], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr


def test_threads_shorter_than_the_state_are_found(walk):
    """The check itself: runs chosen without regard to the taps read the state
    from threads that do not write it, at 4 taps and more."""
    r = subprocess.run([walk, "old"], capture_output=True, text=True, timeout=60)
    assert r.returncode == 1 and r.stdout.startswith("K 4 "), r.stdout
