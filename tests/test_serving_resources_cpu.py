"""Register, scratch and LDS budgets of the serving operators' kernels (no GPU),
from the compiler's resource report under the library's own flags: windows and
the prefix's parts keep the waves per SIMD that their grids assume (four at D = 64,
three at D = 128), with at most a few values spilled around the key loop."""
import concurrent.futures as cf
import re

import pytest

from test_resources_cpu import _num, _parse, _report

SOURCES = ["fa_window.hip", "fa_prefix.hip", "fa_append.hip"]


@pytest.fixture(scope="module")
def reports(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("serving_resources"))
    with cf.ThreadPoolExecutor(len(SOURCES)) as ex:
        texts = dict(zip(SOURCES, ex.map(lambda s: _report(s, d), SOURCES)))
    return {s: (t, _parse(t)) for s, t in texts.items()}


def test_budgets(reports):
    prefill = others = 0
    for src, (text, kernels) in reports.items():
        assert "failed to meet occupancy target" not in text, src
        for name, k in kernels.items():
            assert k["Dynamic Stack"] == "False" and _num(k, "SGPRs Spill") == 0, name
            scratch, occ, lds = (_num(k, "ScratchSize [bytes/lane]"), _num(k, "Occupancy [waves/SIMD]"),
                                 _num(k, "LDS Size [bytes/block]"))
            m = re.search(r"prefill_kernelI.*?Li(64|128)ELi4E", name)
            if not m:
                others += 1
                assert scratch == 0 and occ >= 8, (name, scratch, occ)
                continue
            prefill += 1
            waves, per_simd = (8, 4) if m.group(1) == "64" else (4, 3)
            assert occ >= per_simd and scratch <= 32, (name, occ, scratch)
            assert 4 * per_simd // waves * lds <= 160 * 1024, (name, lds)
    assert prefill >= 40 and others >= 10
