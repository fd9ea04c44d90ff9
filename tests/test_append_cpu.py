"""Refusals of fa_kvcache_append and its paged form: every one is decided on
the host, before any HIP call, so made-up addresses do (no GPU)."""
import ctypes

import pytest

from paper_2608_18656_amd import _lib

M = 1 << 24   # made-up, 16-byte aligned "device" addresses, 16 MiB apart
GOOD = dict(k=M, v=2 * M, kc=3 * M, vc=4 * M, q=5 * M, qo=6 * M, lens=7 * M, table=8 * M, B=2, Hq=4, Hkv=2, N=3,
            Nk=64, D=64, qs=0, ks=0, vs=0, dtype=0, ps=64, mp=2, np=8)
ROT = dict(inv_freq=9 * M, positions=None, rot_dim=64, interleaved=0, axes=1, pair_axis=())


def rotary(**over):
    p = dict(ROT, **over)
    r = _lib.Rotary(p["inv_freq"], p["positions"], p["rot_dim"], p["interleaved"], p["axes"])
    for j, ax in enumerate(p["pair_axis"]):
        r.pair_axis[j] = ax
    return r


def append(rot=None, paged=False, **over):
    p = dict(GOOD, **over)
    lib = _lib.load()
    at = ctypes.addressof(rot) if rot is not None else None
    ptrs = [p["k"], p["v"], p["kc"], p["vc"], p["q"], p["qo"], p["lens"]]
    tail = [p["qs"], p["ks"], p["vs"], at, None, p["dtype"]]
    if paged:
        return lib.fa_kvcache_append_paged(*ptrs, p["table"], p["B"], p["Hq"], p["Hkv"], p["N"], p["D"], p["ps"],
                                           p["mp"], p["np"], *tail)
    return lib.fa_kvcache_append(*ptrs, p["B"], p["Hq"], p["Hkv"], p["N"], p["Nk"], p["D"], *tail)


REFUSED = [
    ({"k": None}, 1), ({"v": None}, 1), ({"kc": None}, 1), ({"vc": None}, 1), ({"lens": None}, 1),
    ({"q": None}, 1), ({"qo": None}, 1),
    ({"B": 0}, 2), ({"N": 0}, 2), ({"Hkv": 0}, 2), ({"Hq": 0}, 2), ({"D": 0}, 2), ({"B": -1}, 2),
    ({"qs": 255}, 2), ({"ks": 120}, 2), ({"vs": -128}, 2),
    ({"B": 1 << 16, "N": 1 << 16}, 2), ({"Hkv": 1 << 22, "Hq": 1 << 22}, 2),
    ({"dtype": 3}, 9), ({"dtype": -1}, 9),
    ({"Hq": 3}, 3),
    ({"D": 60}, 4), ({"D": 264}, 4),
    ({"k": M + 8}, 7), ({"vc": 4 * M + 2}, 7), ({"qo": 6 * M + 4}, 7), ({"lens": 7 * M + 2}, 7),
    ({"qs": 260}, 7), ({"ks": 132}, 7), ({"dtype": 2, "vs": 130}, 7),
    ({"qo": 5 * M + 64}, 8), ({"kc": M + 16}, 8), ({"vc": 3 * M + 1024}, 8), ({"qo": 3 * M}, 8), ({"qo": 2 * M}, 8),
    ({"lens": 6 * M + 16}, 8),
    ({"qs": 512, "qo": 5 * M}, 8),   # in place, but not dense
]


@pytest.mark.parametrize("over,code", REFUSED)
def test_refusals(over, code):
    assert append(**over) == code
    assert append(rot=rotary(), **over) == code
    assert append(paged=True, **over) == code


@pytest.mark.parametrize("over,code", [({"Nk": 0}, 2), ({"Nk": -5}, 2), ({"B": 1 << 30, "N": 1, "Nk": 1 << 30}, 2)])
def test_refusals_contiguous(over, code):
    assert append(**over) == code


@pytest.mark.parametrize("over,code", [
    ({"table": None}, 1), ({"ps": 0}, 2), ({"ps": 65}, 2), ({"ps": 32}, 2), ({"mp": 0}, 2), ({"np": 0}, 2),
    ({"ps": 1 << 20, "mp": 1 << 12}, 2), ({"table": 8 * M + 2}, 7), ({"table": 3 * M}, 8), ({"table": 6 * M + 64}, 8),
])
def test_refusals_paged(over, code):
    assert append(paged=True, **over) == code


@pytest.mark.parametrize("over,code", [
    ({"inv_freq": None}, 1),
    ({"rot_dim": 0}, 14), ({"rot_dim": 3}, 14), ({"rot_dim": 66}, 14), ({"rot_dim": -2}, 14),
    ({"axes": 0}, 14), ({"axes": 5, "positions": 10 * M}, 14), ({"axes": 2}, 14),
    ({"axes": 2, "positions": 10 * M, "pair_axis": (0, 1, 2)}, 14),
    ({"inv_freq": 9 * M + 2}, 7), ({"positions": 10 * M + 1}, 7),
    ({"inv_freq": 6 * M + 16}, 8), ({"positions": 3 * M + 16}, 8), ({"axes": 2, "positions": 4 * M - 40}, 8),
])
def test_refusals_of_the_rotation(over, code):
    assert append(rot=rotary(**over)) == code
    assert append(rot=rotary(**over), paged=True) == code


def test_more_tokens_than_a_grid_takes_are_refused():
    far = {n: (i + 1) << 44 for i, n in enumerate(("k", "v", "kc", "vc", "q", "qo", "lens", "table"))}
    for B, N in (((1 << 25) + 1, 1), (1 << 13, (1 << 12) + 1), (1, 1 << 30)):
        for paged in (False, True):
            assert append(paged=paged, B=B, N=N, mp=1, **far) == 2
