"""csrc/row_part.h: rows that begin anywhere are read in 16-byte loads that stay inside their tensor.  (Compiled here with the host compiler; beam selection reads its logits so.)"""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1811_02084_b200", "csrc")
RUN = 128                                                             # pieces that a warp copies at a time


@pytest.fixture(scope="module")
def whole_pieces(tmp_path_factory):
    d = tmp_path_factory.mktemp("row_part")
    (d / "w.cpp").write_text('#include "row_part.h"\nextern "C" int whole(long long at, int n, long long total, int words, int aligned) { return mtf::whole_pieces(at, n, total, words, aligned); }\n')
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "w.so"), str(d / "w.cpp")], check=True)
    f = ctypes.CDLL(str(d / "w.so")).whole
    f.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return f


@pytest.mark.parametrize("words", [4, 8])                             # f32, bf16
def test_no_load_leaves_the_tensor_and_none_is_given_up_without_need(whole_pieces, words):
    for n in list(range(1, 70)) + [1003, 1024, 1025, 2049, 4099, 50257]:
        for rows in (1, 2, 3, 5, 8, 9, 16, 17):
            total, aligned = rows * n, n % words == 0
            for row in range(rows):
                at = row * n
                off = at % words
                assert off == 0 or not aligned
                whole, full = whole_pieces(at, n, total, words, aligned), n // words
                loads = 1 if aligned else 2
                # the last word that reading piece p takes in, and how far a run's copy goes
                last = lambda p: at - off + (p + loads) * words                          # noqa: E731
                assert 0 <= whole <= full
                assert whole == 0 or last(whole - 1) <= total, (n, rows, row)
                assert whole == full or last(whole) > total, (n, rows, row)
                runs = whole // RUN
                assert at - off + (runs * RUN + (1 if off else 0)) * words <= total or runs == 0


def test_the_selection_reads_its_rows_so():
    text = open(os.path.join(CSRC, "beam_select.cu")).read()
    part = text[text.index("struct Part {"):]
    part = part[:part.index("\n};\n")]
    assert "whole = mtf::whole_pieces(at, n, total, kN, kAligned);" in part and part.count("whole =") == 1
    assert "kAligned ? p[0] : Words<T>::shifted(p[0], p[1], off)" in part and "p < whole ? at(base + p) : load_some(" in part


def test_rows_whose_last_piece_had_a_load_behind_the_tensor(whole_pieces):
    """One row of 50257 words in bf16, 1 x 10, and the last of 5 rows of 9 in f32: they begin on 16 bytes, and the 16 behind their last whole piece are not all theirs."""
    assert [whole_pieces(at, n, total, words, 0) for at, n, total, words in ((0, 50257, 50257, 8), (0, 10, 10, 8), (36, 9, 45, 4))] == [6281, 0, 1]
