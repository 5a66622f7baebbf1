"""Spans that one (first, end) per row cannot say are refused, and what documents do
to prefixes."""

import pytest

pytest.importorskip("torch")

from paper_2512_04013_amd.runtime import row_spans  # noqa: E402


def test_a_window_and_a_prefix_are_refused():
    # row 8 of 9 keys with a window of 2 and a prefix of 4 would see 0 .. 3 and 7 .. 8
    with pytest.raises(ValueError, match="not one span"):
        row_spans([0, 1], [9], window=2, prefix_len=[4])
    with pytest.raises(ValueError, match="window"):
        row_spans([0, 1], [9], window=-1)
    first, end = row_spans([0, 1], [9], window=0, prefix_len=[4])
    assert first.tolist() == [0] and end.tolist() == [9]


def test_documents_cut_a_prefix():
    # one request of five rows: a document of three with a prefix of two, then one of two
    first, end = row_spans([0, 5], [5], prefix_len=[2], doc_start=[0, 0, 0, 3, 3])
    assert first.tolist() == [0, 0, 0, 3, 3] and end.tolist() == [2, 2, 3, 4, 5]
