"""How the waves of the attention kernels meet over tiles in LDS (csrc/hp_meet.hpp, the kernels' own code), on the CPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    exe, csrc = tmp_path_factory.mktemp("meet") / "walk_meet", os.path.join(ROOT, "paper_2605_27678_amd", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-Wall", "-pthread",
                        "-I", csrc, os.path.join(ROOT, "tests", "walk_meet.cpp"), "-o", str(exe)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return lambda *args: subprocess.run([str(exe), *args], capture_output=True, text=True, timeout=300)


def test_every_wave_waits_for_its_own_loads(walk):
    r = walk("loads", "0")
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_waits_by_the_loads_of_other_waves_are_found(walk):
    """64 rows of 96 channels are 768 pieces for 512 lanes: half the waves make one load of a matrix, half two."""
    r = walk("loads", "1")
    assert r.returncode == 1 and "before it is there" in r.stdout, r.stdout + r.stderr


def test_a_flag_is_read_by_all_waves_before_any_goes_on(walk):
    r = walk("flag", "0")
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_a_flag_read_behind_one_barrier_alone_is_found(walk):
    r = walk("flag", "1")
    assert r.returncode == 1 and "read another flag" in r.stdout, r.stdout + r.stderr
