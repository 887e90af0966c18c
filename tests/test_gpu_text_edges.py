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


# ---------------------------------------------------------------------------------------------------------------
# what lies between the rows stays
# ---------------------------------------------------------------------------------------------------------------
def _gapped(values, front, back):
    """The values in rows between gaps of a pattern, and a check that the gaps, a row above and a row below still hold it."""
    rows, cols = values.shape
    wide = torch.full((rows + 2, front + cols + back), 77.0, dtype=values.dtype, device="cuda")
    inner = wide[1:rows + 1, front:front + cols]
    inner.copy_(values)

    def untouched():
        w = wide.clone()
        w[1:rows + 1, front:front + cols] = 77.0
        return bool((w == 77.0).all())
    return inner, untouched


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("acc", [False, True])
@pytest.mark.parametrize("M,V,dim", [(1, 3, 1), (5, 9, 7), (300, 40, 33), (513, 20, 264), (2048, 9, 130), (2049, 300, 131), (20_000, 500, 9), (40_000, 700, 13), (40_000, 3000, 257)])
def test_embed_bwd_writes_its_rows_alone(M, V, dim, acc, odt):
    gen = torch.Generator(device="cuda").manual_seed(M + dim)
    g = torch.randint(-2, 3, (M, dim), generator=gen, device="cuda").float()                # whole values: exact in any order
    ids = (torch.rand(M, generator=gen, device="cuda") ** 4 * (V + 2)).to(torch.int32) - 1
    for front, back in ((0, 1), (1, 0), (3, 2), (8, 8)):
        out, untouched = _gapped(torch.ones((V, dim), dtype=odt, device="cuda"), front, back)
        kge.embed_bwd(g, ids, V, out=out, accumulate=acc)
        ok = (ids >= 0) & (ids < V)
        want = torch.full((V, dim), 1.0 if acc else 0.0, device="cuda").index_add_(0, ids[ok].long(), g[ok])
        assert torch.equal(out, want.to(odt)) and untouched()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("acc", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 1, 100), (3, 30, 300), (20, 17, 200), (70, 131, 260), (200, 97, 4200), (1030, 1029, 200), (300, 1700, 1300), (4353, 3841, 130)])
def test_matmul_writes_its_rows_alone(m, n, k, acc, dt):
    """Every kernel and the launch that adds up splits: rows and columns behind the last whole tile, group of four and of eight."""
    gen = torch.Generator(device="cuda").manual_seed(m + n + k)
    a, b = (kge.quantize(torch.randint(-1, 2, (r, k), generator=gen, device="cuda").float()) for r in (m, n))
    plain = kge.matmul_quantized(a, b, dtype=F32)
    for front, back in ((0, 1), (1, 0), (3, 2), (8, 8)):
        out, untouched = _gapped(torch.ones((m, n), dtype=dt, device="cuda"), front, back)
        kge.matmul_quantized(a, b, out=out, accumulate=acc)
        assert torch.equal(out, (plain + 1.0 if acc else plain).to(dt)) and untouched()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (130, 64), (5, 767), (40, 8193), (40_000, 1001)])
def test_dropout_and_lookup_write_their_rows_alone(rows, cols, dt):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, r = (torch.randn((rows, cols), generator=gen, device="cuda").to(dt) for _ in range(2))
    ids = torch.randint(-1, rows + 1, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    d = kge.Dropout(0.3, 5)
    for front, back in ((0, 1), (1, 0), (3, 2), (8, 8)):
        xs, rs = _gapped(x, back, front)[0], _gapped(r, 5, 0)[0]
        for res, gapped in ((None, None), (r, rs)):
            out, untouched = _gapped(torch.ones((rows, cols), dtype=dt, device="cuda"), front, back)
            kge.dropout(xs, d, residual=gapped, out=out)
            assert torch.equal(out, kge.dropout(x, d, residual=res)) and untouched()
        out, untouched = _gapped(torch.ones((rows, cols), dtype=dt, device="cuda"), front, back)
        kge.embed(xs, ids, dropout=d, out=out)
        assert torch.equal(out, kge.embed(x, ids, dropout=d)) and untouched()


# ---------------------------------------------------------------------------------------------------------------
# gradient: three digits, numbers that are not finite
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M,V", [(20_000, 20_000_000), (40_000, 80_000_000)])
def test_embed_bwd_sorts_in_three_passes(M, V):
    """Parts of 2^17 rows, by eight bits at a time, of collected and of dealt out ids."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    pool = torch.randint(0, V, (M // 3,), generator=gen, device="cuda")
    ids = pool[torch.randint(0, M // 3, (M,), generator=gen, device="cuda")]
    ids[::50], ids[1::50], ids[2::50], ids[3::50] = 0, V - 1, -1, V // 2                    # runs of whole chunks
    ids = ids.to(torch.int32)
    g = torch.randint(-3, 4, (M, 1), generator=gen, device="cuda").float()
    ok = ids >= 0
    got = kge.embed_bwd(g, ids, V)
    assert torch.equal(got, torch.zeros((V, 1), device="cuda").index_add_(0, ids[ok].long(), g[ok]))
    ones = torch.ones((V, 1), device="cuda")
    assert torch.equal(kge.embed_bwd(g, ids, V, out=ones, accumulate=True), got + 1)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("M,V", [(400, 30), (1500, 30), (9000, 300), (40_000, 300)])
def test_embed_bwd_of_numbers_that_are_not_finite(M, V, dt):
    """NaN and infinities in a live element reach their row and column alone; in a dropped one and at a padded position they reach nothing."""
    dim, p = 24, 0.5
    gen = torch.Generator(device="cuda").manual_seed(M)
    ids = (torch.rand(M, generator=gen, device="cuda") ** 3 * V).to(torch.int32)
    ids[::9] = -1
    ids[::11] = V
    g = torch.randint(-2, 3, (M, dim), generator=gen, device="cuda").to(dt)
    d = kge.Dropout(p, 3, step=2, tag=1)
    kept = kge.dropout(torch.ones((M, dim), device="cuda"), d) > 0
    dead = ~kept | (ids < 0).unsqueeze(1) | (ids >= V).unsqueeze(1)
    clean = kge.embed_bwd(g, ids, V, dropout=d)
    for bad in (float("nan"), float("inf"), -float("inf")):
        assert torch.equal(kge.embed_bwd(torch.where(dead, torch.full_like(g, bad), g), ids, V, dropout=d), clean)
        live = (~dead).nonzero()[::97]
        x = g.clone()
        x[live[:, 0], live[:, 1]] = bad
        want = clean.clone()
        want[ids[live[:, 0]].long(), live[:, 1]] = bad
        assert torch.equal(torch.nan_to_num(kge.embed_bwd(x, ids, V, dropout=d), 1e9, 2e9, -2e9), torch.nan_to_num(want, 1e9, 2e9, -2e9))


# ---------------------------------------------------------------------------------------------------------------
# in front of the path
# ---------------------------------------------------------------------------------------------------------------
def test_entities_from_an_8_bit_feature_table_through_the_loss():
    """e = e_S + D o (M e_F) of a step's slots, with e_F in 8 bits and gathered by the product, through kge_loss_bwd, whose gradient rows come back as a dense one
    of e_S.  The front part against 64 bits, the loss and its gradient against the same call on entities made in 64 bits and rounded."""
    n_ent, n_rel, d, f, B, N = 400, 5, 64, 200, 96, 160
    gen = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")                                          # noqa: E731
    e_s, m, rel = rand(n_ent, d) * 0.3, rand(d, f) * 0.05, rand(n_rel, d) * 0.3
    feat, proj = kge.quantize(rand(n_ent, f)), kge.quantize(m)
    ids = torch.randint(0, n_ent, (2 * B + N,), generator=gen, device="cuda", dtype=torch.int32)
    r = torch.randint(0, n_rel, (B,), generator=gen, device="cuda", dtype=torch.int32)
    slot = torch.arange(2 * B + N, dtype=torch.int32, device="cuda")
    drop = kge.Dropout(0.25, 7, step=3, tag=12)
    e = kge.dropout(kge.matmul_quantized(feat, proj, rows=ids, dtype=F32), drop, residual=kge.embed(e_s, ids))

    def values(q):
        v = q.codes.view(FLOAT8[q.fmt]).double()
        return v * torch.exp2(q.scales[:, :v.shape[1] // 128].double() - 127).repeat_interleave(128, dim=1)
    kept = (kge.dropout(torch.ones((2 * B + N, d), device="cuda"), drop) > 0).double() / 0.75
    p, mag = (x[ids.long()] @ y.t() for x, y in ((values(feat), values(proj)), (values(feat).abs(), values(proj).abs())))
    want = e_s[ids.long()].double() + kept * p
    # (256 products in any order, factor, its product, sum)
    assert bool(((e.double() - want).abs() <= kept * mag * (256 + 3) * 2.0 ** -24 + want.abs() * 2.0 ** -24).all())

    def loss(x):
        return kge.loss_bwd(kge.Model("distmult", x, rel), "logsigmoid", slot[:B], r, slot[B:2 * B], slot[2 * B:], gamma=2.0)
    got, ref = loss(e), loss(want.float())
    assert torch.equal(got["g_ent_idx"], slot)
    for key in ("loss", "g_ent", "g_rel"):
        # e is off by 256 * 2^-24 = 1.5e-5 of its terms at most; what comes out is smooth in it, and a call's own sums are good to 1e-5
        assert float((got[key] - ref[key]).double().norm()) <= 1e-4 * float(ref[key].double().norm()), key
    dense = kge.embed_bwd(got["g_ent"], ids, n_ent)
    zero = torch.zeros((n_ent, d), dtype=torch.float64, device="cuda")
    sums, sizes = (zero.index_add(0, ids.long(), x) for x in (got["g_ent"].double(), got["g_ent"].double().abs()))
    count = torch.bincount(ids.long(), minlength=n_ent).unsqueeze(1)
    assert bool(((dense.double() - sums).abs() <= sizes * count * 2.0 ** -24).all())
