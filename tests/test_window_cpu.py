"""Refusals of fa_fwd_window and its paged form, decided on the host before any
HIP call, and the workspace sizes (no GPU)."""
import pytest

from paper_2608_18656_amd import _lib, window_workspace_bytes, workspace_bytes

M = 1 << 24
GOOD = dict(q=M, k=2 * M, v=3 * M, o=4 * M, lse=5 * M, lens=6 * M, table=7 * M, B=2, Hq=4, Hkv=2, Nq=1, Nk=128, D=64,
            ps=64, mp=2, np=8, window=16, sinks=4, scale=0.125, it=0, ot=0, ws=8 * M, wb=1 << 22)


def window(paged, **over):
    p = dict(GOOD, **over)
    lib = _lib.load()
    head = [p["q"], p["k"], p["v"], p["o"], p["lse"], p["lens"]]
    tail = [p["window"], p["sinks"], p["scale"], None, p["it"], p["ot"], p["ws"], p["wb"]]
    if paged:
        return lib.fa_fwd_window_paged(*head, p["table"], p["B"], p["Hq"], p["Hkv"], p["Nq"], p["D"], p["ps"], p["mp"],
                                       p["np"], *tail)
    return lib.fa_fwd_window(*head, p["B"], p["Hq"], p["Hkv"], p["Nq"], p["Nk"], p["D"], *tail)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("over,code", [
    ({"window": 0}, 15), ({"window": -1}, 15), ({"sinks": -1}, 15),
    ({"q": None}, 1), ({"o": None}, 1), ({"B": 0}, 2), ({"Hq": 3}, 3), ({"D": 60}, 4), ({"Nq": 129}, 5),
    ({"scale": float("inf")}, 6), ({"k": 2 * M + 8}, 7), ({"lens": 6 * M + 2}, 7), ({"o": M}, 8), ({"o": 6 * M}, 8),
    ({"lse": 4 * M}, 8), ({"it": 3}, 9), ({"ot": 1}, 9),
    ({"ws": None}, 1), ({"ws": 8 * M + 8}, 7), ({"wb": 16}, 10), ({"ws": 4 * M}, 8), ({"ws": 3 * M}, 8),
])
def test_refusals(paged, over, code):
    assert window(paged, **over) == code


@pytest.mark.parametrize("over,code", [
    ({"table": None}, 1), ({"lens": None}, 1), ({"ps": 96}, 2), ({"mp": 0}, 2), ({"np": 0}, 2), ({"it": 2, "ot": 2}, 9),
    ({"D": 96}, 4), ({"table": 4 * M}, 8),
])
def test_refusals_paged(over, code):
    assert window(True, **over) == code


def test_workspace_sizes():
    a = (16, 32, 8, 1, 8192, 128)
    need = window_workspace_bytes(*a, 1024, "bf16", sinks=4)
    assert 0 < need <= workspace_bytes(*a, "bf16")
    assert need == workspace_bytes(16, 32, 8, 1, 1028, 128, "bf16")
    assert window_workspace_bytes(*a, 1 << 40, "bf16", sinks=1 << 40) == workspace_bytes(*a, "bf16")
    assert window_workspace_bytes(16, 32, 8, 512, 8192, 128, 1024, "bf16") == 0   # row blocks for all CUs: no parts
    assert window_workspace_bytes(1, 32, 8, 8, 8192, 96, 1024, "bf16") == 0 and window_workspace_bytes(1, 2, 2, 9, 500, 64, 100, "f32") == 0
    few = window_workspace_bytes(1, 32, 8, 8, 8192, 128, 4096, "bf16", sinks=4)
    assert few > 0
    for Nk in (8, 100, 4000, 4105, 8191):
        assert window_workspace_bytes(1, 32, 8, 8, Nk, 128, 4096, "bf16", sinks=4) <= few
    assert window_workspace_bytes(*a, 0, "bf16") == 0 and window_workspace_bytes(*a, 5, "bf16", sinks=-1) == 0
    for Nk in (1, 700, 1027, 1029, 5000):
        assert window_workspace_bytes(16, 32, 8, 1, Nk, 128, 1024, "bf16", sinks=4) <= need


def test_workspace_apart_from_lengths_and_table():
    assert window(False, ws=6 * M) == 8 and window(True, ws=6 * M) == 8 and window(True, ws=7 * M) == 8
