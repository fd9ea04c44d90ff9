"""Caches whose last tile would end past 2^31 keys: the kernels count keys in ints, so
these are refused on the host before any HIP call (no GPU; made-up addresses).  Small
heads make such caches possible: 2^31 keys of 8 fp16 columns are 34 GB."""
import pytest

from paper_2608_18656_amd import _lib, validate

A = [(i + 1) << 44 for i in range(9)]
MOST = 2**31 - 256


def window(Nq, Nk, D, it=0, lens=A[5], B=1, Hq=1, Hkv=1):
    return _lib.load().fa_fwd_window(*A[:5], lens, B, Hq, Hkv, Nq, Nk, D, 100, 4, 0.5, None, it, it, A[6], 1 << 30)


@pytest.mark.parametrize("Nk", [MOST + 1, 2**31 - 128, 2**31 - 1])
@pytest.mark.parametrize("Nq,D,it", [(1, 8, 0), (3, 8, 1), (1, 64, 2), (1, 64, 0), (7, 64, 1), (1, 128, 1)])
def test_windows(Nk, Nq, D, it):
    assert window(Nq, Nk, D, it) == 2 and window(Nq, Nk, D, it, lens=None) == 2


@pytest.mark.parametrize("Nq,D,it", [(1, 8, 0), (3, 64, 1), (1, 96, 2)])
def test_all_keys(Nq, D, it):
    lib = _lib.load()
    for Nk in (MOST + 1, 2**31 - 1):
        assert lib.fa_fwd(*A[:5], 1, 1, 1, Nq, Nk, D, 0, 0.5, None, it, it) == 2
        assert lib.fa_fwd_kvcache(*A[:5], A[5], 1, 1, 1, Nq, Nk, D, 0, 0.5, None, it, it) == 2
        assert validate(*A[:5], 1, 1, 1, Nq, Nk, D, 0, 0.5, it) == 2
    assert validate(*A[:5], 1, 1, 1, Nq, MOST, D, 0, 0.5, it) == 0


def test_decode_takes_them():
    """To the end of its last chunk of 32."""
    assert validate(*A[:5], 1, 1, 1, 1, 2**31 - 32, 64, 0, 0.5, "f16") == 0
    assert validate(*A[:5], 1, 1, 1, 1, 2**31 - 31, 64, 0, 0.5, "f16") == 2


@pytest.mark.parametrize("Nq", [1, 9])
def test_windows_of_pages(Nq):
    lib = _lib.load()
    args = [*A[:5], A[7], A[8], 1, 1, 1, Nq, 64, 64, 2**25 - 1, 1, 2**31 - 1, 4, 0.5, None, 0, 0, A[6], 1 << 30]
    assert lib.fa_fwd_window_paged(*args) == 2


def test_pages_of_long_rows():
    """Key rows past the 16-bit kernels' offsets go to the fp32-weight kernel."""
    far = [(i + 1) << 52 for i in range(8)]
    lib = _lib.load()
    for call, tail in ((lib.fa_fwd_kvcache_paged, []), (lib.fa_fwd_window_paged, [far[7], 1 << 30])):
        args = [*far[:7], 1, 1 << 19, 1 << 19, 3, 128, 64, 2**25 - 1, 1] + ([100, 4] if tail else [1]) + [0.5, None, 0, 0] + tail
        assert call(*args) == 2
