"""The plans of attentions over sequences, under sanitizers: what a launch reads, the largest launches and their grids."""
import os

from test_sanitizers import NATIVE, ROOT, SAN, build_and_run


def test_sequence_plans_under_sanitizers(tmp_path):
    exe = str(tmp_path / "seq_plan_check")
    build_and_run(["g++", "-std=c++17", *SAN, "-o", exe, os.path.join(NATIVE, "seq_plan_check.cpp"),
                   os.path.join(ROOT, "paper_2609_23286_amd", "csrc", "rv_seq.cpp")], exe, "sequence plans OK")
