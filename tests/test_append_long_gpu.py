"""kvcache_append of long prompts, past the size (96 MB read and written) from which
the inputs are read by non-temporal loads: every type, both pairings, whole and
partial chunks, pages, a number of tokens that no workgroup's share divides.  The
reference and the tolerance are those of test_append_gpu."""
import pytest
import torch

import paper_2608_18656_amd as fa

import test_append_gpu as short

pytestmark = pytest.mark.gpu

HELD = 96 << 20

CASES = [   # as test_append_gpu.CASES
    (1, 4097, 32, 8, 128, 128, False, 1, "f16", 0, 4200, [4099]),         # the next token count past the limit
    (2, 2051, 32, 8, 128, 128, True, 3, "bf16", 64, 2112, [2100, 2051]),
    (3, 1367, 32, 8, 128, 0, False, 1, "bf16", 0, 1400, [1400, 1367, 900]),   # no rotation, padding
    (1, 4097, 32, 8, 64, 64, False, 1, "f32", 256, 4352, [4200]),
    (1, 4099, 16, 4, 128, 24, True, 4, "f32", 0, 4099, [4099]),
    (1, 7299, 32, 8, 72, 24, False, 1, "f16", 64, 7360, [7350]),          # halves of 12 columns, element by element
    (1, 5963, 16, 4, 88, 34, False, 1, "f32", 0, 6000, [5970]),
    (1, 5963, 16, 4, 88, 34, True, 2, "f32", 0, 6000, [5990]),
    (1, 7299, 32, 8, 72, 20, True, 1, "bf16", 0, 7300, [7300]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:11]))
def test_append(case):
    B, N, Hq, Hkv, D, dt = case[0], case[1], case[2], case[3], case[4], case[8]
    assert 2 * B * N * (Hq + 2 * Hkv) * D * (4 if dt == "f32" else 2) > HELD
    short.test_append(case, True)


@pytest.mark.parametrize("rot", [128, 40])
def test_in_place(rot):
    N, Hq, Hkv, D = 4100, 32, 8, 128
    q, k, v = (torch.randn((1, N, h, D), device="cuda").half() for h in (Hq, Hkv, Hkv))
    caches = [torch.zeros((1, N, Hkv, D), device="cuda").half() for _ in range(4)]
    n = torch.tensor([N], dtype=torch.int32, device="cuda")
    freq = (1e4 ** (-torch.arange(0, rot, 2) / rot)).float().cuda()
    out = fa.kvcache_append(k, v, caches[0], caches[1], n, q=q, inv_freq=freq)
    mine = q.clone()
    assert fa.kvcache_append(k, v, caches[2], caches[3], n, q=mine, q_out=mine, inv_freq=freq) is mine
    torch.cuda.synchronize()
    assert torch.equal(out, mine) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
