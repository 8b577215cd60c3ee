"""Where few new tokens' logits and sums lie in LDS (csrc/st3_block_few.h), on the host: vectors of 16 bytes are aligned for every number of rows."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_parts_are_apart_and_aligned(tmp_path):
    exe = str(tmp_path / "few_lds")
    root = os.path.join(HERE, "..")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2412_20105_amd", "csrc"),
                    os.path.join(HERE, "few_lds_driver.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
