"""fwd_prefix_paged where every sequence is shorter than the shared prefix (it is
still being read in, say): what lies in the shared pages behind the longest one is
NaN here and has no part in the result, in parts and in one pass.

The reference and the tolerance are those of test_prefix_gpu."""
import pytest
import torch

import paper_2608_18656_amd as fa

from test_prefix_gpu import check_case

pytestmark = pytest.mark.gpu

PARTS = [
    # B, Hq, Hkv, Nq, Np, Nk, D, dt, causal, lens, page
    (4, 16, 2, 1, 8192, 64, 64, "f16", True, [8000, 4096, 0, 63], 64),
    (4, 16, 2, 1, 8192, 0, 64, "bf16", False, [8000, 4096, 0, 63], 256),
    (3, 32, 8, 1, 4096, 128, 128, "bf16", True, [33, 1, 0], 64),
    (3, 32, 8, 1, 4096, 128, 128, "f16", False, [4095, 2048, 31], 64),
    (2, 8, 2, 40, 4096, 128, 128, "bf16", True, [3000, 17], 64),      # fewer keys than queries
    (2, 8, 2, 40, 4096, 128, 64, "f16", False, [1000, 0], 128),
    (64, 8, 1, 1, 2048, 64, 128, "bf16", True, [3 + 7 * b for b in range(64)], 64),   # row blocks of their own lengths
    (3, 8, 2, 1, 4096, 64, 64, "f16", True, [0, 0, -5], 64),          # nobody has a key
]
ONE_PASS = [
    (12, 16, 1, 1, 64, 64, 64, "bf16", False, [5 * b for b in range(12)], 64),
    (2, 8, 2, 31, 128, 64, 64, "f16", True, [100, 0], 64),
    (2, 8, 2, 32, 128, 64, 128, "bf16", True, [127, 20], 64),
]


def in_parts(B, Hq, Hkv, Nq, Np, Nk, D, dt, causal, lens, page):
    """Whether the call takes partial results, and with them a workspace."""
    pool = torch.zeros((1, page, Hkv, D), dtype={"f16": torch.float16, "bf16": torch.bfloat16}[dt], device="cuda")
    table = torch.zeros((B, (Np + Nk) // page), dtype=torch.int32, device="cuda")
    q = torch.zeros((B, Nq, Hq, D), dtype=pool.dtype, device="cuda")
    try:
        fa.fwd_prefix_paged(q, pool, pool.clone(), table, torch.tensor(lens, dtype=torch.int32, device="cuda"), Np,
                            causal=causal, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    except fa.FaError as e:
        assert e.status == 10
        return True
    return False


@pytest.mark.parametrize("parts,case", [(True, c) for c in PARTS] + [(False, c) for c in ONE_PASS],
                         ids=lambda c: c if isinstance(c, bool) else "-".join(str(x) for x in c[:9]) + f"-{c[10]}")
def test_all_shorter_than_the_prefix(parts, case):
    assert max(case[9]) < case[4]
    assert in_parts(*case) == parts
    check_case(*case)
