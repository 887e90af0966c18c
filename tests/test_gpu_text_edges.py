"""Uses of the text side's calls at their edges: two host threads on one stream, rows between gaps, sorts of three passes, numbers that are not finite and
numbers at the ends of the scales' range.  Tolerances count roundings: eps / 2 of the output's type, 2^-24 for every fp32 operation."""
import threading

import numpy as np
import pytest
import torch

import paper_2211_12281_amd as kge

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def test_two_threads_on_one_stream():
    """Gradients over lists of different lengths and tables, and products split along k, from two host threads on torch's default stream, both without a
    workspace: the results of the same calls one after the other."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")                                          # noqa: E731
    grads = [(rand(M, d), (torch.rand(M, generator=gen, device="cuda") ** 5 * V).to(torch.int32), V) for M, V, d in
             [(40_000, 90, 64), (3_000, 70_000, 24), (90_000, 20_000, 8), (33_000, 5, 40)]]
    mats = [(kge.quantize(rand(m, k)), kge.quantize(rand(n, k))) for m, n, k in [(130, 140, 6000), (300, 90, 9000)]]
    calls = [lambda a=a: kge.embed_bwd(*a) for a in grads] + [lambda m=m: kge.matmul_quantized(*m, dtype=F32) for m in mats]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    got, errors, gate = {0: [], 1: []}, [], threading.Barrier(2, timeout=60)

    def work(t):
        try:
            gate.wait()
            for i in range(40):
                k = (5 * i if t else i) % len(calls)
                got[t].append((k, calls[k]()))
        except Exception as e:                                  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(t,)) for t in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for k, out in got[0] + got[1]:
        assert torch.equal(out, want[k])


@pytest.mark.parametrize("p", [0.0, 0.5])
@pytest.mark.parametrize("dt,odt", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -2.0])
def test_padded_positions_are_zeros_whatever_the_scale(scale, dt, odt, p):
    table = torch.randn((4, 23), device="cuda").to(dt)
    ids = torch.tensor([0, -1, 4, 3, -2**31, 2**31 - 1], dtype=torch.int32, device="cuda")
    out = kge.embed(table, ids, scale=scale, dropout=kge.Dropout(p, 1) if p else None, dtype=odt).float()
    dead = out[[1, 2, 4, 5]]
    assert not bool(dead.any()) and not bool(torch.signbit(dead).any())
    if not p:
        assert torch.equal(torch.nan_to_num(out[[0, 3]], 7.0), torch.nan_to_num((table[[0, 3]].float() * scale).to(odt).float(), 7.0))
