"""Splits of a window's single tokens: as many as a cache of the visible keys gets,
at both head sizes, and the result past the size where there are several (GPU; the
reference and the tolerance are those of test_window_gpu)."""
import pytest

from paper_2608_18656_amd import window_workspace_bytes, workspace_bytes


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 32, 8), (1, 16, 1), (16, 16, 16)])
def test_as_a_cache_of_the_visible_keys(B, Hq, Hkv, D):
    for window, sinks in ((1, 0), (500, 4), (700, 4), (1024, 4), (1148, 4), (1149, 4), (5000, 64)):
        assert window_workspace_bytes(B, Hq, Hkv, 1, 16384, D, window, "f16", sinks=sinks) == \
            workspace_bytes(B, Hq, Hkv, 1, window + sinks, D, "f16")


@pytest.mark.gpu
@pytest.mark.parametrize("case", [
    (1, 8, 2, 1, 3000, 64, "f16", 513, 0, [2999], 0),
    (1, 32, 8, 1, 4096, 64, "bf16", 700, 4, [4093], 64),
    (3, 16, 1, 1, 2500, 64, "f16", 1024, 4, [2500, 1027, 0], 0),
    (2, 8, 8, 1, 3000, 64, "bf16", 1000, 152, [3000, 1153], 128),
    (2, 4, 4, 1, 1300, 64, "f16", 1152, 0, None, 0),
], ids=lambda c: "-".join(str(x) for x in c[:9]) + f"-{c[10]}")
def test_tokens(case):
    from test_window_gpu import check_case

    check_case(*case)
