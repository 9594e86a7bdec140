"""Exponent bytes of an 8-bit cache are copied by aligned words of four: the last one ends where the array does."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2605_22718_b200.build import CSRC, ROOT, _nvcc


@pytest.fixture(scope="module")
def words(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    out = str(tmp_path_factory.mktemp("host") / "libwords.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", cuda, "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "exponent_words.cc"), "-o", out], check=True)
    fn = C.CDLL(out).exponent_words
    fn.argtypes, fn.restype = [C.c_uint32] * 3, C.c_uint32
    return fn


@pytest.mark.parametrize("n", [*range(1, 41), 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 1, *range(2 ** 32 - 5, 2 ** 32)])
def test_every_word_lies_in_the_array_and_holds_its_byte(words, n):
    assert words(n, 0, min(n, 64)) == 0 and words(n, n - min(n, 64), min(n, 64)) == 0
