"""The streaming example end to end: compression passes, attention over the live
half and over quantised pages, and how far the two answers are apart.

With random keys of unit variance the scores' spread is that of the queries
(scale 1/sqrt(dim) times sqrt(dim)), so thousands of rows share the weight. A
group of 64 normal values spans about 4.8 of their standard deviations: 4-bit
values are off by 4.8 / 15 / sqrt(12) = 0.09 of one, 8-bit ones by 0.0055. That
error enters once by V (its mean over the weights, like the output itself) and
once by the scores (off by 0.09, which changes weights by that much of
themselves): together sqrt(2) of it, 0.13 and 0.008, plus bf16's roundings of the
two outputs, 0.003. Allowed: 1.5 times that."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import stream_answer  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,allowed", [("u4", 0.2), ("u8", 0.016)])
def test_the_stream_is_answered(fmt, allowed):
    r = stream_answer.run(fmt=fmt, layers=2, heads=2, share=3, dim=64, grid=6, cap=16, keep=10, step=2, frames=30, question=9,
                          answer=5, page=16)
    assert r["passes"] == 3 and r["finite"]          # at 16 frames, then every 6
    assert r["rows"] == 12 * 36 + 9 + 5
    assert 0 < r["distance"] < allowed


def test_the_7b_shape():
    r = stream_answer.run(fmt="u8", frames=64)
    assert r["passes"] == 2 and r["rows"] == 32 * 196 + 31 and r["finite"] and 0 < r["distance"] < 0.016
