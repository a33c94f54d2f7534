"""Which operands share memory (csrc/spans.hpp), in a host program that compares it with looking at every byte."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_spans_against_every_byte(tmp_path):
    exe = str(tmp_path / "spans")
    build = subprocess.run(["g++", "-O2", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined,signed-integer-overflow",
                            "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2402_11857_amd", "csrc"), "-o", exe,
                            os.path.join(ROOT, "tests", "host", "spans.cpp")], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "spans ok" in run.stdout, run.stdout + run.stderr
