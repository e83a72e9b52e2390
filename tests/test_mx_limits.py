"""Limits of the MXFP4 entry points that the header states, as host code sees them (no GPU)."""
import os
import re

import pytest

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_largest_norm_is_the_same_in_header_and_binding():
    from paper_1609_07228_amd import efanna
    header = open(os.path.join(ROOT, "include", "efanna.h")).read()
    stated = re.search(r"#define EFANNA_MX_MAX_NORM (\S+)f\b", header)
    assert stated and float(stated.group(1)) == efanna.MX_MAX_NORM == 2.0 ** 126
