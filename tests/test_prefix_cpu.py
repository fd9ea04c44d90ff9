"""Refusals of fa_fwd_prefix and its paged form, decided on the host before any
HIP call, and the workspace sizes (no GPU)."""
import pytest

from paper_2608_18656_amd import _lib, prefix_workspace_bytes

M = 1 << 24
GOOD = dict(q=M, kp=2 * M, vp=3 * M, k=4 * M, v=5 * M, o=6 * M, lse=7 * M, lens=8 * M, table=9 * M, B=2, Hq=4, Hkv=2, Nq=1,
            Np=8000, Nk=64, D=64, ps=64, mp=126, np=200, pl=8000, causal=1, scale=0.125, it=0, ot=0, ws=10 * M, wb=1 << 22)


def prefix(paged, **over):
    p = dict(GOOD, **over)
    lib = _lib.load()
    tail = [p["causal"], p["scale"], None, p["it"], p["ot"], p["ws"], p["wb"]]
    if paged:
        return lib.fa_fwd_prefix_paged(p["q"], p["k"], p["v"], p["o"], p["lse"], p["lens"], p["table"], p["B"], p["Hq"],
                                       p["Hkv"], p["Nq"], p["D"], p["ps"], p["mp"], p["np"], p["pl"], *tail)
    return lib.fa_fwd_prefix(p["q"], p["kp"], p["vp"], p["k"], p["v"], p["o"], p["lse"], p["lens"], p["B"], p["Hq"],
                             p["Hkv"], p["Nq"], p["Np"], p["Nk"], p["D"], *tail)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("over,code", [
    ({"q": None}, 1), ({"k": None}, 1), ({"o": None}, 1), ({"B": 0}, 2), ({"Nq": 0}, 2), ({"Hq": 3}, 3),
    ({"D": 60}, 4), ({"D": 96}, 4), ({"Nq": 8065}, 5), ({"scale": float("nan")}, 6), ({"v": 5 * M + 8}, 7),
    ({"lens": 8 * M + 2}, 7), ({"o": M}, 8), ({"o": 8 * M}, 8), ({"lse": 6 * M}, 8), ({"lse": 4 * M}, 8), ({"it": 3}, 9),
    ({"ot": 1}, 9), ({"it": 2, "ot": 2}, 9), ({"B": 1 << 20, "Nq": 1 << 12, "causal": 0}, 2),
    ({"ws": None}, 1), ({"ws": 10 * M + 8}, 7), ({"wb": 64}, 10), ({"ws": 6 * M}, 8), ({"ws": 5 * M}, 8), ({"ws": 8 * M}, 8),
])
def test_refusals(paged, over, code):
    assert prefix(paged, **over) == code


@pytest.mark.parametrize("over,code", [
    ({"kp": None}, 1), ({"vp": None}, 1), ({"Np": 0}, 2), ({"Nk": 0}, 2), ({"Np": 1 << 30}, 2), ({"kp": 2 * M + 8}, 7),
    ({"o": 2 * M}, 8), ({"lse": 3 * M}, 8), ({"ws": 3 * M}, 8),
])
def test_refusals_contiguous(over, code):
    assert prefix(False, **over) == code


@pytest.mark.parametrize("over,code", [
    ({"table": None}, 1), ({"lens": None}, 1), ({"ps": 96}, 2), ({"mp": 0}, 2), ({"np": 0}, 2), ({"pl": 0}, 2),
    ({"pl": 100}, 2), ({"pl": 64 * 127}, 2), ({"pl": -64}, 2), ({"table": 9 * M + 2}, 7), ({"table": 6 * M}, 8), ({"ws": 9 * M}, 8),
])
def test_refusals_paged(over, code):
    assert prefix(True, **over) == code


def test_workspace_sizes():
    need = prefix_workspace_bytes(64, 32, 8, 1, 8192, 1024, 128, "bf16")
    row = 64 * 32 * 130 * 4
    assert need >= 2 * row and need % row == 0
    for Np, Nk in ((1, 1), (63, 1024), (4000, 17), (8191, 1000), (8192, 0)):
        assert 0 < prefix_workspace_bytes(64, 32, 8, 1, Np, Nk, 128, "bf16") <= need
    assert prefix_workspace_bytes(64, 32, 8, 64, 8192, 1024, 128, "bf16") == 0   # full waves on a full chip: one pass
    for over in (dict(B=0), dict(Hq=3, Hkv=2), dict(D=96), dict(Np=0), dict(Nk=-1), dict(Np=1 << 30), dict(in_dtype="f32"),
                 dict(B=1 << 30, Nq=1 << 30)):
        a = dict(B=2, Hq=4, Hkv=2, Nq=1, Np=100, Nk=100, D=64, in_dtype="f16")
        a.update(over)
        assert prefix_workspace_bytes(**a) == 0


def test_key_rows_past_32_bit_offsets_are_refused():
    far = {n: (i + 1) << 44 for i, n in enumerate(("q", "kp", "vp", "k", "v", "o", "lse", "lens", "table", "ws"))}
    for D, last in ((128, 270600), (64, 266304)):
        for paged in (False, True):
            assert prefix(paged, Hq=last + 1, Hkv=last + 1, B=1, D=D, Np=8000, wb=1 << 50, **far) == 2
