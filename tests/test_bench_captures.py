"""The DRAM traffic that bench.py reports comes from captures of particular kernel sources; they are reported only while the digests agree."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("bench_module", os.path.join(ROOT, "bench.py"))
bench = importlib.util.module_from_spec(spec)
spec.loader.exec_module(bench)


@pytest.mark.parametrize("op", sorted(bench.NCU_CAPTURES))
def test_captures_belong_to_the_sources(op):
    assert bench.NCU_CAPTURES[op][3] == bench.csrc_digest(op)
