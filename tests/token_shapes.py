"""Asks csrc/token_plan.hpp which forms it chooses, through tests/token_shapes.cpp."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
TILES = ("BIG", "MID", "HALF", "SMALL", "SMALL_SPLIT")


def ask(folder, questions):
    """A number for each question, as tests/token_shapes.cpp reads them."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    exe = os.path.join(str(folder), "token_shapes")
    if not os.path.exists(exe):
        subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(HERE, "token_shapes.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], input="\n".join(" ".join(map(str, q)) for q in questions), capture_output=True, text=True, check=True)
    return [int(x) for x in r.stdout.split()]
