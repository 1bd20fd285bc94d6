"""Rules of the kernels that are launched while the one before them in the stream
ends, read off their sources (no GPU): each waits for that one, and none reads
through the path for data that is constant while the kernel lives, as the lengths,
tables and rows that it reads may be that kernel's results."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_00535_gb300", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    text = re.sub(r"//[^\n]*", "", text)
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


FILES = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "early_launch()" in source(f))


def test_there_are_such_files():
    assert {"pages.cu", "window.cu", "window_tc.cu"} <= set(FILES)


@pytest.mark.parametrize("name", FILES)
def test_every_kernel_waits_for_the_one_before(name):
    text = source(name)
    starts = [m.start() for m in re.finditer(r"\b__global__\b", text)]
    assert starts
    for a, b in zip(starts, starts[1:] + [len(text)]):
        assert "after_previous();" in text[a:b], text[a:a + 200]


@pytest.mark.parametrize("name", FILES)
def test_no_kernel_reads_through_the_constant_path(name):
    headers = re.findall(r'#include "(\w+\.cuh)"', open(os.path.join(CSRC, name)).read())
    for f in [name] + headers:
        text = source(f)
        assert "__ldg(" not in text and "ld.global.nc" not in text and "ld.const" not in text, f
        assert "__restrict__" not in text, f  # (with it the compiler may choose that path by itself)
