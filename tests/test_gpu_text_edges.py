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


FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m", [16, 1280])                       # (few rows, tiles)
@pytest.mark.parametrize("side", ["a", "b"])
@pytest.mark.parametrize("fmt,exact", [("e4m3", range(3, 247)), ("e5m2", range(10, 240))])
def test_product_of_every_code_under_scales_from_end_to_end(fmt, exact, side, m, dt):
    """One code times a power of two that brings it back into range.  fp32 output: exact under the bytes of `exact`; below them the element is rounded to a
    multiple of 2^-133 (off by half of one), above them infinite from 2^128 on.  bf16 output: exact, as such a product has four bits at most."""
    codes = torch.zeros((1280, 128), dtype=torch.uint8, device="cuda")
    codes[:, 5] = (torch.arange(1280, device="cuda") % 256).to(torch.uint8)
    value = codes[:256, 5].cpu().view(FLOAT8[fmt]).double()
    ones = torch.zeros((1280, 128), dtype=torch.uint8, device="cuda")
    ones[:, 5] = 0x38                                           # 1 in e4m3
    for s in (*range(0, 14), 120, 127, *range(236, 255)):
        t = min(254 - s, 246)                                   # (code * 2^(s + t - 254): in range)
        scales = [torch.zeros((1280, 4), dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales[0][:, 0], scales[1][:, 0] = s, t
        q, one = kge.Quantized(codes, scales[0], 128, fmt), kge.Quantized(ones[:m], scales[1][:m], 128)
        got = kge.matmul_quantized(q, one, dtype=dt)[:256, 0] if side == "a" else kge.matmul_quantized(one, q, dtype=dt)[0, :256]
        got, element, want = got.double().cpu(), value * 2.0 ** (s - 127), value * 2.0 ** (s + t - 254)
        assert torch.equal(torch.isnan(got), torch.isnan(want)), s
        ok = torch.isfinite(want)
        if dt == F32:
            big = ok & (element.abs() >= 2.0 ** 128)
            assert torch.equal(got[big], want[big] * float("inf")) and (not bool(big.any()) or s > exact[-1])
            ok &= ~big
            tol = torch.zeros_like(want) if s in exact or s > exact[-1] else torch.full_like(want, 2.0 ** -134 * 2.0 ** (t - 127))
        else:
            tol = torch.zeros_like(want)                        # (four bits times a power of two)
        assert bool(((got - want).abs() <= tol)[ok].all()), s


def _cancelling(m, n, k):
    """64 * 64 - 64 * 64 + 2^-3 beside zeros, in different places of the rows: 2^-3 whatever the order of fp32 sums."""
    a, b = torch.zeros((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    a[:, 0], a[:, 1], a[:, 2], b[:, 0], b[:, 1], b[:, 2] = 64, 64, 0.5, 64, -64, 0.25
    return kge.quantize(a), kge.quantize(b)


@pytest.mark.parametrize("m,n,k", [(1, 300, 100), (16, 4096, 1000), (40, 300, 700), (300, 700, 900), (1100, 900, 260), (140, 500, 4100), (4100, 4090, 300)])
def test_bf16_output_with_fp32_sums(m, n, k):
    """The sums of the fp32 output, rounded once, from every kernel: few rows, tiles, split and whole, large tiles; gathered and added too."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    a, b = (kge.quantize(torch.randn((r, k), generator=gen, device="cuda")) for r in (m, n))
    assert torch.equal(kge.matmul_quantized(a, b, fp32_sums=True), kge.matmul_quantized(a, b, dtype=F32).to(BF16))
    rows = torch.randint(-1, m + 1, (m,), generator=gen, device="cuda", dtype=torch.int32)
    got = kge.matmul_quantized(a, b, rows=rows, fp32_sums=True, out=torch.ones((m, n), dtype=BF16, device="cuda"), accumulate=True)
    assert torch.equal(got, (kge.matmul_quantized(a, b, rows=rows, dtype=F32) + 1).to(BF16))
    assert torch.equal(kge.matmul_quantized(a, b, dtype=F32, fp32_sums=True), kge.matmul_quantized(a, b, dtype=F32))
    a, b = _cancelling(m, n, k)
    assert bool((kge.matmul_quantized(a, b, fp32_sums=True) == 0.125).all())
    assert bool(((kge.matmul_quantized(a, b).float() - 0.125).abs() <= 7 * 2.0 ** -13 * 4096).all())
