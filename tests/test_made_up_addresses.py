"""Where a GPU can be seen, no test hands made-up addresses to a call that is not refused."""
from __future__ import annotations

import types

from tests import conftest


def item(nodeid, *keywords):
    marks = []
    return types.SimpleNamespace(nodeid=nodeid, keywords=keywords, add_marker=marks.append, marks=marks)


def test_they_are_skipped_there(monkeypatch):
    for gpu in (True, False):
        monkeypatch.setattr(conftest, "_gpu_available", lambda: gpu)
        items = [item("tests/test_paged_q4.py::test_row_calls_and_copy_refusals"), item("tests/test_paged_q4.py::test_decode_refusals[kw0-1]"),
                 item("tests/test_paged_q4.py::test_copy[64]", "gpu")]
        conftest.pytest_collection_modifyitems(None, items)
        assert [len(x.marks) for x in items] == ([1, 0, 0] if gpu else [0, 0, 1])
