"""Paged sequences and prepared projections without a GPU: the page lists and attention passes under
sanitizers, and the refusals of every entry point."""
import os

from test_sanitizers import NATIVE, ROOT, SAN, build_and_run


def test_page_lists_and_passes_under_sanitizers(tmp_path):
    exe = str(tmp_path / "seq_logic_check")
    build_and_run(["g++", "-std=c++17", *SAN, "-o", exe, os.path.join(NATIVE, "seq_logic_check.cpp"),
                   os.path.join(ROOT, "paper_2609_23286_amd", "csrc", "rv_seq.cpp")], exe, "sequence logic OK")
