"""Host functions of the paged 4-bit cache's sources, compiled by themselves with g++ so that tests can ask them directly."""
from __future__ import annotations

import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_27646_amd", "csrc")


def between(name: str, first: str, last: str) -> str:
    """The text of a source file from `first` up to `last`, which is left out."""
    text = open(os.path.join(CSRC, name)).read()
    start = text.index(first)
    return text[start:text.index(last, start)]


def compiled(folder, code: str) -> ctypes.CDLL:
    """`code` as a library, device annotations taken away."""
    head = "#include <algorithm>\n#include <cstdint>\n#include <cstdlib>\n#include \"hqmq_cache4.h\"\n" + "".join(
        f"#define {word} {meaning}\n" for word, meaning in (("__device__", ""), ("__host__", ""), ("__forceinline__", "inline")))
    source, lib = os.path.join(folder, "host.cpp"), os.path.join(folder, "host.so")
    with open(source, "w") as f:
        f.write(head + code)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-o", lib, source], check=True)
    return ctypes.CDLL(lib)
