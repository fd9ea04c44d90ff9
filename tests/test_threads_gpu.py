"""Host threads that call on one stream at a time, without a workspace of their own:
every call gives the bits that it gives alone (calls whose partial results share the
stream's one buffer, with other numbers of parts and rows)."""
import threading

import pytest
import torch

import paper_2608_18656_amd as fa

pytestmark = pytest.mark.gpu


def calls():
    gen = torch.Generator(device="cuda").manual_seed(11)

    def r(*shape):
        return torch.randn(shape, generator=gen, device="cuda").half()

    q, k, v = r(2, 1, 16, 128), r(2, 5000, 4, 128), r(2, 5000, 4, 128)
    few = r(2, 6, 16, 128)
    kp, vp, ks, vs, q4 = r(3000, 4, 64), r(3000, 4, 64), r(4, 90, 4, 64), r(4, 90, 4, 64), r(4, 1, 32, 64)
    n = torch.tensor([5000, 3100], dtype=torch.int32, device="cuda")
    return [lambda: fa.fwd_kvcache(q, k, v, n),
            lambda: fa.fwd_window(q, k, v, 3000, sinks=4, seqlens_k=n),
            lambda: fa.fwd_window(few, k, v, 4000, sinks=4, seqlens_k=n),
            lambda: fa.fwd_prefix(q4, kp, vp, ks, vs, causal=True),
            lambda: fa.fwd_splitkv_noalloc(q, k, v, 7)]


def test_one_stream():
    fs = calls()
    alone = [f() for f in fs]
    torch.cuda.synchronize()
    got, errors = [[] for _ in fs], []

    def caller(i):
        try:
            for _ in range(60):
                got[i].append(fs[i]())
        except Exception as e:   # noqa: BLE001 (a thread's exception would be lost)
            errors.append(e)

    threads = [threading.Thread(target=caller, args=(i,)) for i in range(len(fs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for ref, results in zip(alone, got):
        assert len(results) == 60
        for o, lse in results:
            assert torch.equal(o, ref[0]) and torch.equal(lse, ref[1])
