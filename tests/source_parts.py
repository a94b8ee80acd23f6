"""Parts of the CUDA sources compiled for the host, so that a test can run their index arithmetic and
rules without a GPU.  Test code only."""

import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_09231_gb300", "csrc")


def part(file, head):
    """The definition in csrc/`file` that starts with `head`, up to its closing brace (and semicolon)."""
    src = open(os.path.join(CSRC, file)).read()
    start = src.index(head)
    assert src.count(head) == 1, head
    j = src.index("{", start) + 1
    depth = 1
    while depth:
        depth += {"{": 1, "}": -1}.get(src[j], 0)
        j += 1
    return src[start:j] + (";" if src[j] == ";" else "")


def run(code, tmp_path, text=""):
    """Standard output of the C++ program `code` with `text` on its standard input."""
    source, program = tmp_path / "part.cpp", tmp_path / "part"
    source.write_text(code)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(program), str(source)], check=True)
    return subprocess.run([str(program)], input=text, check=True, capture_output=True, text=True).stdout
