"""The tokens that a work-group takes of packed sequences, over the host's offsets and over any others that the device may hold: the kernels'
own rules (csrc/packed_spans.hpp), compiled for the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2605_08696_amd", "csrc")


def test_spans_lie_inside_the_operands_whatever_the_offsets(tmp_path):
    program = str(tmp_path / "packed_spans")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC,
                    os.path.join(HERE, "packed_spans.cpp"), "-o", program], check=True, timeout=120)
    done = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0 and done.stdout == "ok\n", done.stdout + done.stderr
