"""Token embeddings, dropout, quantisation and the quantised matrix product against plain implementations in 64 bits on the CPU.

Tolerances count roundings: eps / 2 of the output's type, 2^-24 for every fp32 operation in front of it."""
import math

import numpy as np
import pytest
import torch

import paper_2211_12281_amd as kge

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
EMAX = {"e4m3": 8, "e5m2": 15}
SEED, STEP, TAG = 0x123456789ABCDEF, 7, 3


def _rng(*key):
    return np.random.default_rng([int(k) for k in key])


def _values(shape, dtype, *key, std=1.0):
    return (torch.from_numpy(_rng(*key).normal(size=shape)) * std).to(dtype)


def _padded(t, pad):
    """The same values on the GPU in rows that are `pad` elements longer, so that they start anywhere."""
    if pad == 0:
        return t.cuda()
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, pad // 2:pad // 2 + t.shape[1]] = t.cuda()
    return wide[:, pad // 2:pad // 2 + t.shape[1]]


def _factor(rows, cols, p, step=STEP, seed=SEED, tag=TAG, row0=0):
    """float64 [rows, cols]: the dropout factors of rows row0 and on, from big-integer arithmetic on each counter block."""
    thr = math.floor(p * 65536 + 0.5)
    out = np.zeros((rows, -(-cols // 8) * 8))
    for r in range(rows):
        for g in range(-(-cols // 8)):
            c, k = [row0 + r, g, step, tag], [seed & 0xFFFFFFFF, seed >> 32]
            for _ in range(10):
                p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                c = [p1 >> 32 ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, p0 >> 32 ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
                k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
            for i in range(8):
                h = c[i // 2] >> 16 * (i % 2) & 0xFFFF
                out[r, 8 * g + i] = 65536 / (65536 - thr) if h >= thr else 0.0
    return torch.from_numpy(out[:, :cols])


def _ids(M, V, *key, pad=True):
    g = _rng(*key)
    ids = np.minimum(g.zipf(1.3, size=M) - 1, V - 1) if V else np.zeros(M)
    if pad and M > 3:
        ids[g.integers(0, M, size=max(1, M // 17))] = -1
        ids[0], ids[1] = V, V - 1                                # one past the end (a padded position too), and the last row
    return torch.from_numpy(ids.astype(np.int32))


def _within(got, want, tol, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


# ---------------------------------------------------------------------------------------------------------------
# lookup
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt,odt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("M,V,dim,pad,p", [(1, 5, 768, 0, 0.0), (7, 1, 1, 0, 0.5), (33, 100, 7, 1, 0.1), (300, 50, 129, 3, 0.25), (17, 1000, 8, 0, 0.9),
                                           (65, 40, 2049, 5, 0.0), (2, 9, 9001, 0, 0.1)])
def test_embed(dt, odt, M, V, dim, pad, p):
    table, ids, scale = _values((V, dim), dt, 1, M, dim), _ids(M, V, 2, M), 1.7
    d = kge.Dropout(p, SEED, STEP, TAG) if p else None
    out = _padded(torch.zeros((M, dim), dtype=odt), pad)
    got = kge.embed(_padded(table, pad), ids.cuda(), scale=scale, dropout=d, out=out)
    assert got is out
    live = ((ids >= 0) & (ids < V)).unsqueeze(1)
    f = _factor(M, dim, p) if p else torch.ones((), dtype=torch.float64)
    want = torch.where(live, table.double()[ids.long().clamp(0, V - 1)] * float(np.float32(scale)) * f, torch.zeros((), dtype=torch.float64))
    _within(got, want, want.abs() * (HALF[odt] + 3 * U), "embed")       # (the factor 2^16 / (2^16 - thr) is rounded to fp32 too)
    if pad:
        assert bool(torch.isnan(out._base[:, 0]).all() if pad > 1 else torch.isnan(out._base[:, -1]).all())   # what lies between the rows stays


def test_embed_keeps_infinities_and_drops_them_whole():
    table = torch.full((2, 64), float("inf"))
    table[1] = float("nan")
    got = kge.embed(table.cuda(), torch.tensor([0, 1, 0], dtype=torch.int32).cuda(), dropout=kge.Dropout(0.5, SEED, STEP, TAG)).cpu()
    f = _factor(3, 64, 0.5)
    assert bool((got[f == 0] == 0).all()) and bool(torch.isinf(got[0][f[0] > 0]).all()) and bool(torch.isnan(got[1][f[1] > 0]).all())


def test_embed_of_an_empty_table_is_zeros():
    out = kge.embed(torch.empty((0, 24), device="cuda"), torch.tensor([0, -1, 5], dtype=torch.int32, device="cuda"))
    assert out.shape == (3, 24) and not bool(out.any())


# ---------------------------------------------------------------------------------------------------------------
# gradient of the lookup
# ---------------------------------------------------------------------------------------------------------------
def _bwd_case(M, V, dim, p, dt, *key, ids=None):
    g = _values((M, dim), dt, 3, M, dim, *key)
    ids = _ids(M, V, 4, M, *key) if ids is None else ids
    scale = 0.7
    f = _factor(M, dim, p) if p else torch.ones((), dtype=torch.float64)
    terms = g.double() * f * float(np.float32(scale))
    live = (ids >= 0) & (ids < V)
    at = ids.long().clamp(0, max(V - 1, 0))[live]
    want, mag = (torch.zeros((V, dim), dtype=torch.float64).index_add_(0, at, x[live]) for x in (terms, terms.abs()))
    n = torch.zeros(V, dtype=torch.float64).index_add_(0, at, torch.ones(at.numel(), dtype=torch.float64)).unsqueeze(1)
    return g, ids, scale, want, mag * (n + 3) * U                       # n terms added in any order; factor, scale and its product


@pytest.mark.parametrize("dt,odt", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("M,V,dim,pad,p,acc", [(1, 7, 768, 0, 0.0, False), (5, 3, 1, 1, 0.5, True), (40, 1, 33, 0, 0.1, False), (700, 64, 72, 3, 0.1, True),
                                               (700, 2000, 257, 1, 0.0, False), (0, 5, 16, 0, 0.0, False), (64, 1, 600, 0, 0.0, True),
                                               (129, 2, 8, 0, 0.25, False), (3000, 300, 24, 0, 0.0, True),
                                               (512, 20, 264, 1, 0.1, False), (513, 20, 264, 1, 0.1, False), (2048, 9, 130, 0, 0.0, False),
                                               (2049, 9, 130, 0, 0.0, True), (4500, 60_000, 16, 0, 0.2, False)])
def test_embed_bwd(dt, odt, M, V, dim, pad, p, acc):
    g, ids, scale, want, tol = _bwd_case(M, V, dim, p, dt)
    old = _values((V, dim), odt, 5, V)
    out = _padded(old, pad)
    got = kge.embed_bwd(_padded(g, pad), ids.cuda(), V, scale=scale, dropout=kge.Dropout(p, SEED, STEP, TAG) if p else None, out=out, accumulate=acc)
    assert got is out
    if acc:
        want = want + old.double()
        tol = tol + want.abs() * U
        none = torch.ones(V, dtype=torch.bool)
        none[ids.long()[(ids >= 0) & (ids < V)]] = False
        assert torch.equal(got.cpu()[none], old[none])                  # rows without a position stay as they are
    _within(got, want, tol + (want.abs() + tol) * HALF[odt], "embed_bwd")


@pytest.mark.parametrize("M,V,dim", [(32768, 700, 40), (32769, 700, 40), (70000, 90000, 24), (70000, 3, 72), (32768, 3_000_000, 8), (40000, 3_000_000, 8),
                                     (530_000, 5000, 8), (33000, 1, 16), (20000, 70_000, 600), (16384, 400, 32), (16385, 400, 32)])
@pytest.mark.parametrize("p", [0.0, 0.1])
def test_embed_bwd_long(M, V, dim, p):
    """Both sorts, runs of thousands of positions, every chunk boundary."""
    g, ids, scale, want, tol = _bwd_case(M, V, dim, p, BF16)
    d = kge.Dropout(p, SEED, STEP, TAG) if p else None
    got = kge.embed_bwd(g.cuda(), ids.cuda(), V, scale=scale, dropout=d)
    _within(got, want, tol + (want.abs() + tol) * U, "embed_bwd")
    assert torch.equal(got, kge.embed_bwd(g.cuda(), ids.cuda(), V, scale=scale, dropout=d))        # the same sums every time


@pytest.mark.parametrize("start,n", [(0, 64), (0, 63), (1, 63), (1, 64), (63, 65), (64, 64), (10, 200), (0, 256)])
@pytest.mark.parametrize("padded", [0, 2100, 17_000])
def test_embed_bwd_runs_against_chunks(start, n, padded):
    """A run of n positions that starts at a given place of the sorted list; with padded positions the call is one of those that take chunks of 8 and of 32."""
    ids = torch.from_numpy(_rng(9, start, n).permutation(np.concatenate([np.zeros(start), np.full(n, 1), np.full(37, 2), np.full(padded, -1)])).astype(np.int32))
    g, ids, scale, want, tol = _bwd_case(ids.numel(), 3, 16, 0.0, F32, 1, ids=ids)
    _within(kge.embed_bwd(g.cuda(), ids.cuda(), 3, scale=scale), want, tol + (want.abs() + tol) * U)


@pytest.mark.parametrize("odt", [F32, BF16])
def test_embed_bwd_past_the_caches(odt):
    """A gradient of 90 MB into 200 MB and more, with rows of odd widths and gaps: whole values, exact in any order."""
    M, V, dim = 45_000, 102_500, 1001
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = torch.randint(-2, 3, (M, dim), generator=gen, device="cuda").to(BF16)
    ids = (torch.rand(M, generator=gen, device="cuda") ** 4 * (V + 1000)).to(torch.int32) - 100
    ids[::3] = 7
    out = torch.full((V, dim + 3), 5.0, dtype=odt, device="cuda")
    kge.embed_bwd(g, ids, V, out=out[:, :dim])
    ok = (ids >= 0) & (ids < V)
    want = torch.zeros((V, dim), dtype=torch.float32, device="cuda").index_add_(0, ids[ok].long(), g[ok].float())
    assert torch.equal(out[:, :dim], want.to(odt)) and bool((out[:, dim:] == 5).all())


def test_embed_bwd_only_padded_positions():
    ids = torch.full((100,), -1, dtype=torch.int32, device="cuda")
    g = torch.full((100, 16), float("nan"), device="cuda")
    out = torch.ones((4, 16), device="cuda")
    kge.embed_bwd(g, ids, 4, out=out, accumulate=True)
    assert bool((out == 1).all())
    assert not bool(kge.embed_bwd(g, ids, 4, out=out).any())


def test_embed_gradient_against_differences():
    """<g, embed(T + e X) - embed(T - e X)> / 2e = <embed_bwd(g), X>: exact up to rounding, as the lookup is linear."""
    M, V, dim, p = 60, 11, 20, 0.25
    d = kge.Dropout(p, SEED, STEP, TAG)
    T, X, g = _values((V, dim), F32, 20), _values((V, dim), F32, 21), _values((M, dim), F32, 22)
    ids, e = _ids(M, V, 23), 0.5
    up, down = (kge.embed((T + s * e * X).cuda(), ids.cuda(), scale=3.0, dropout=d).double().cpu() for s in (1, -1))
    lhs = float((g.double() * (up - down)).sum() / (2 * e))
    G = kge.embed_bwd(g.cuda(), ids.cuda(), V, scale=3.0, dropout=d).double().cpu()
    rhs = float((G * X.double()).sum())
    mag = float((g.double().abs() * (up.abs() + down.abs())).sum() / (2 * e)) + float((G.abs() * X.double().abs()).sum())
    assert abs(lhs - rhs) <= mag * (M + 8) * U


# ---------------------------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad,p,res", [(1, 1, 0, 0.5, False), (3, 767, 0, 0.1, True), (130, 64, 1, 0.25, True), (5, 9, 3, 0.999, False),
                                                 (2, 8200, 0, 0.1, True), (40, 256, 0, 0.0, True), (9, 7, 2, 0.99999, True)])
def test_dropout(dt, rows, cols, pad, p, res):
    x, r = _values((rows, cols), dt, 30, rows), _values((rows, cols), dt, 31, rows)
    thr = min(math.floor(float(np.float32(p)) * 65536 + 0.5), 65535)
    f = _factor(rows, cols, thr / 65536)
    out = kge.dropout(_padded(x, pad), kge.Dropout(p, SEED, STEP, TAG), residual=_padded(r, pad) if res else None)
    want = x.double() * f
    tol = want.abs() * 2 * U
    if res:
        want = want + r.double()
        tol = tol + want.abs() * U
    _within(out, want, tol + (want.abs() + tol) * HALF[dt], "dropout")
    if p == 0.0:
        assert torch.equal(out.cpu(), (x.float() + r.float()).to(dt))


def test_dropout_rate_and_independence():
    """Kept share of 4M elements within five standard deviations, other seeds, steps and tags give other masks, neighbours are uncorrelated."""
    x = torch.ones((4096, 1024), device="cuda")
    masks = [kge.dropout(x, kge.Dropout(0.3, *k)) > 0 for k in [(1, 0, 0), (2, 0, 0), (1, 1, 0), (1, 0, 1)]]
    n, keep = x.numel(), 1 - round(0.3 * 65536) / 65536
    for m in masks:
        assert abs(float(m.double().mean()) - keep) <= 5 * math.sqrt(keep * (1 - keep) / n)
    both = [(masks[0], masks[i]) for i in (1, 2, 3)] + [(masks[0][:, :-1], masks[0][:, 1:]), (masks[0][:-1], masks[0][1:])]
    for a, c in both:
        assert abs(float((a & c).double().mean()) - keep ** 2) <= 5 * math.sqrt(keep ** 2 * (1 - keep ** 2) / a.numel())


def test_dropout_in_place_and_infinities():
    x = _values((50, 100), BF16, 33).cuda()
    x[:, 3], x[:, 4] = float("inf"), float("nan")
    r = _values((50, 100), BF16, 34).cuda()
    d = kge.Dropout(0.5, SEED, STEP, TAG)
    want = kge.dropout(x, d, residual=r)
    same = lambda got: torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(want, 7.0))   # noqa: E731
    x2, r2 = x.clone(), r.clone()
    assert same(kge.dropout(x2, d, residual=r, out=x2)) and same(kge.dropout(x, d, residual=r2, out=r2))
    dropped = _factor(50, 100, 0.5) == 0
    assert torch.equal(want.cpu()[dropped], r.cpu()[dropped])


def test_dropout_gradient_is_the_same_call():
    x, g = _values((20, 33), F32, 35), _values((20, 33), F32, 36)
    d, f = kge.Dropout(0.4, SEED, STEP, TAG), _factor(20, 33, round(0.4 * 65536) / 65536)
    got = kge.dropout(g.cuda(), d)
    _within(got, g.double() * f, (g.double() * f).abs() * 3 * U)
    up, down = (kge.dropout((x + s * 0.5 * g).cuda(), d).double().cpu() for s in (1, -1))
    lhs = float((g.double() * (up - down)).sum())
    rhs = float((got.double().cpu() * g.double()).sum())
    mag = float((g.double().abs() * (up.abs() + down.abs())).sum())
    assert abs(lhs - rhs) <= mag * 8 * U


# ---------------------------------------------------------------------------------------------------------------
# quantisation
# ---------------------------------------------------------------------------------------------------------------
def _decode(codes, fmt):
    """Values of all codes from the format's definition: sign, exponent, mantissa."""
    eb, mb = (4, 3) if fmt == "e4m3" else (5, 2)
    bias = 2 ** (eb - 1) - 1
    c = np.arange(256)
    e, m = c >> mb & (2 ** eb - 1), c & (2 ** mb - 1)
    v = np.where(e > 0, (1 + m / 2 ** mb) * 2.0 ** (e - bias), m / 2 ** mb * 2.0 ** (1 - bias))
    if fmt == "e4m3":
        v[(c & 127) == 127] = np.nan
    else:
        v[e == 31] = np.where(m[e == 31] == 0, np.inf, np.nan)
    return torch.from_numpy(np.where(c >> 7, -v, v))[codes.long()]


def _quantize(x, fmt):
    """(codes' values float64 [rows, 128 blocks], scales uint8) of x by rows, one block after the other."""
    rows, cols = x.shape
    nb, mb, emin = -(-cols // 128), 3 if fmt == "e4m3" else 2, -6 if fmt == "e4m3" else -14
    v = np.zeros((rows, nb * 128))
    v[:, :cols] = x.double().numpy()
    s = np.zeros((rows, -(-nb // 4) * 4), dtype=np.uint8)
    for r in range(rows):
        for k in range(nb):
            blk = v[r, 128 * k:128 * k + 128]
            fin = np.abs(blk[np.isfinite(blk)])
            top = fin.max() if fin.size else 0.0
            if top > 0:
                e = -127
                while top > 1.75 * 2.0 ** (EMAX[fmt] + e):
                    e += 1
                s[r, k] = e + 127
            u = blk * 2.0 ** (127 - int(s[r, k]))
            with np.errstate(divide="ignore", invalid="ignore"):
                step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(u))), emin) - mb)
                q = np.where(np.isfinite(u), np.rint(u / step) * step, u)
            if fmt == "e4m3":
                q = np.where(np.isinf(u), np.nan, q)
            v[r, 128 * k:128 * k + 128] = q
    return torch.from_numpy(v), torch.from_numpy(s)


def _same(q, x, fmt):
    want, scales = _quantize(x, fmt)
    assert torch.equal(q.scales.cpu(), scales)
    got = _decode(q.codes.cpu(), fmt)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, 0.0, 1e9, -1e9), torch.nan_to_num(want, 0.0, 1e9, -1e9))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 128, 0), (5, 129, 1), (130, 7, 3), (128, 128, 0), (257, 300, 1), (2, 700, 0), (129, 513, 5)])
def test_quantize(dt, fmt, rows, cols, pad):
    x = _values((rows, cols), dt, 40, rows, cols) * torch.from_numpy(10.0 ** _rng(41).uniform(-3, 3, size=(rows, 1))).to(dt)
    row, col = kge.quantize(_padded(x, pad), fmt=fmt, by="both")
    _same(row, x, fmt)
    _same(col, x.t(), fmt)
    for q, one in ((row, kge.quantize(_padded(x, pad), fmt=fmt)), (col, kge.quantize(_padded(x, pad), fmt=fmt, by="col"))):
        assert torch.equal(q.codes, one.codes) and torch.equal(q.scales, one.scales)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_every_binade_and_special_values(fmt):
    """Ties, subnormal codes, blocks of zeros, subnormal and largest fp32 numbers, infinities and NaN in one block that keeps the others' scale."""
    x = torch.zeros((12, 256))
    x[0, :128] = torch.arange(128) * 2.0 ** -9
    x[0, 127] = 448.0                                                   # scale 1 in e4m3: codes 2^-9 apart below 2^-6, ties between them
    x[1, :100] = (torch.arange(100) + 0.5) * 2.0 ** -9
    x[1, 101] = -448.0
    x[2, 0], x[2, 1] = 1e-45, -3e-39                                    # subnormal fp32 numbers
    x[3, 0], x[3, 1] = torch.finfo(F32).max, -1e30
    x[4, 0], x[4, 1], x[4, 2], x[4, 3], x[4, 130] = float("inf"), -float("inf"), float("nan"), 0.3, 2.0
    x[5, 5] = float("nan")
    x[6] = -0.0
    x[7, :8] = torch.tensor([1.75, 1.7500001, 3.5, -3.5000002, 448.0, 448.00003, 57344.0, -57348.0])
    x[8, 0] = 1.0
    x[9, :128], x[9, 128:] = 464.0, 465.0
    x[10] = torch.from_numpy(2.0 ** _rng(44).uniform(-40, 0, size=256))
    x[11] = torch.from_numpy(2.0 ** _rng(45).uniform(-149, -120, size=256))
    row, col = kge.quantize(x.cuda(), fmt=fmt, by="both")
    _same(row, x, fmt)
    _same(col, x.t(), fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_writes_its_rows_alone(fmt):
    x = _values((9, 200), F32, 46).cuda()
    big = torch.full((9, 512), 0xAB, dtype=torch.uint8, device="cuda")
    sc = torch.full((9, 16), 0xCD, dtype=torch.uint8, device="cuda")
    q = kge.Quantized(big[:, :256], sc[:, 4:8], 200, fmt)
    kge.quantize(x, fmt=fmt, out=q)
    plain = kge.quantize(x, fmt=fmt)
    assert torch.equal(big[:, :256], plain.codes) and torch.equal(sc[:, 4:8], plain.scales)
    assert bool((big[:, 256:] == 0xAB).all()) and bool((sc[:, :4] == 0xCD).all()) and bool((sc[:, 8:] == 0xCD).all())


# ---------------------------------------------------------------------------------------------------------------
# matrix product
# ---------------------------------------------------------------------------------------------------------------
def _dequantized(q):
    v = _decode(q.codes.cpu(), q.fmt)
    return v * 2.0 ** (q.scales.cpu()[:, :v.shape[1] // 128].double().repeat_interleave(128, dim=1) - 127)


def _product(a, b, rows, dtype):
    """(product in 64 bits, bound of its error): fp32 sums of k products in any order; the 8-bit instructions besides align groups of eight
    products to the largest of them and drop what lies 2^-13 below it, seven times per group at most (the block's largest |a| times its largest
    |b| bounds that product)."""
    A, B = _dequantized(a), _dequantized(b)
    if rows is not None:
        ok = (rows >= 0) & (rows < A.shape[0])
        A = torch.where(ok.unsqueeze(1), A[rows.long().clamp(0, max(A.shape[0] - 1, 0))] if A.shape[0] else torch.zeros((rows.numel(), A.shape[1]), dtype=torch.float64),
                        torch.zeros((), dtype=torch.float64))
    k = A.shape[1]
    tol = (A.abs() @ B.abs().t()) * (k + 8) * 2 * U
    if dtype == BF16 and k:
        top = [x.abs().view(x.shape[0], k // 128, 128).amax(dim=2) for x in (A, B)]
        tol = tol + (top[0] @ top[1].t()) * (128 - 16) * 2.0 ** -13
    return A @ B.t(), tol


def _q(rows, cols, fmt, *key, std=1.0):
    x = _values((rows, cols), F32, 50, *key, std=std) * torch.from_numpy(2.0 ** _rng(51, *key).integers(-3, 4, size=(rows, 1))).float()
    return kge.quantize(x.cuda(), fmt=fmt)


SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 300), (16, 33, 129), (17, 40, 1000), (33, 100, 257), (64, 15, 2048), (65, 130, 128), (100, 64, 384),
          (128, 128, 640), (129, 257, 100), (300, 200, 2500), (70, 70, 5000), (513, 300, 130), (1000, 3, 260), (66, 1, 127), (3, 5, 0), (80, 90, 0),
          # beyond what workgroups of few rows take: tiles, split and whole, with rows and columns behind the last whole one; one token of many columns
          (1025, 1030, 130), (1100, 900, 260), (40, 9000, 100), (140, 500, 4100), (30, 700, 7000), (2100, 2000, 0), (1, 8200, 2000), (13, 9000, 300), (1, 9000, 5000)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_matmul(dt, fa, fb, m, n, k):
    a, b = _q(m, k, fa, m, k, 1), _q(n, k, fb, n, k, 2)
    got = kge.matmul_quantized(a, b, dtype=dt)
    want, tol = _product(a, b, None, dt)
    _within(got, want, tol + (want.abs() + tol) * HALF[dt], "matmul")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("fa,fb,m,n,k", [("e4m3", "e4m3", 4100, 4090, 300), ("e5m2", "e4m3", 4096, 4096, 128), ("e4m3", "e5m2", 65_600, 130, 700),
                                         ("e5m2", "e5m2", 4353, 3841, 1100)])
def test_matmul_large_tiles(dt, fa, fb, m, n, k):
    """256 tiles of 256 x 256 and more: whole ones, rows and columns behind the last whole one, one to nine blocks; gathered, added, into rows with gaps."""
    a, b = _q(4500, k, fa, 10, k), _q(n, k, fb, 11, k)
    rows = torch.from_numpy(_rng(56, m).integers(-2, 4502, size=m).astype(np.int32))
    want, tol = _product(a, b, rows, dt)
    got = kge.matmul_quantized(a, b, rows=rows.cuda(), dtype=dt)
    _within(got, want, tol + (want.abs() + tol) * HALF[dt], "matmul")
    old = torch.ones((m, n), dtype=dt)
    out = _padded(old, 3)
    kge.matmul_quantized(a, b, rows=rows.cuda(), out=out, accumulate=True)
    want += 1
    tol += want.abs() * U
    _within(out, want, tol + (want.abs() + tol) * HALF[dt], "matmul")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,n,k,pad", [(5, 30, 300, 1), (90, 131, 260, 3), (200, 96, 4200, 2), (1, 7, 128, 0), (1030, 1029, 200, 3), (300, 1700, 1300, 1)])
def test_matmul_gathered_accumulated_strided(dt, m, n, k, pad):
    a, b = _q(50, k, "e4m3", m, 3), _q(n, k, "e4m3", n, 4)
    rows = torch.from_numpy(_rng(52, m).integers(0, 50, size=m).astype(np.int32))
    if m > 4:
        rows[1], rows[2], rows[4] = -1, 50, 49
    old = _values((m, n), dt, 53)
    out = _padded(old, pad)
    kge.matmul_quantized(a, b, rows=rows.cuda(), out=out, accumulate=True)
    want, tol = _product(a, b, rows, dt)
    want = want + old.double()
    tol = tol + want.abs() * U
    _within(out, want, tol + (want.abs() + tol) * HALF[dt], "matmul")
    got = kge.matmul_quantized(a, b, rows=rows.cuda(), dtype=dt)
    if m > 4:
        assert not bool(got[[1, 2]].any()) and torch.equal(out.cpu()[[1, 2]], old[[1, 2]])


def test_matmul_gathers_nothing_from_an_empty_table():
    b = _q(20, 256, "e4m3", 5)
    for m in (70, 70_000):
        out = kge.matmul_quantized(kge.Quantized.empty(0, 256), b, rows=torch.zeros(m, dtype=torch.int32, device="cuda"), dtype=F32)
        assert out.shape == (m, 20) and not bool(out.any())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,n", [(3, 30), (70, 30), (1100, 1000), (5000, 4100)])
def test_matmul_nan_stays_in_its_row(dt, m, n):
    x, w = _values((m, 200), F32, 54), _values((n, 200), F32, 55)
    x[1, 7], w[4, 100] = float("nan"), float("nan")
    got = kge.matmul_quantized(kge.quantize(x.cuda()), kge.quantize(w.cuda()), dtype=dt).cpu()
    want = torch.zeros((m, n), dtype=torch.bool)
    want[1], want[:, 4] = True, True
    assert torch.equal(torch.isnan(got), want)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,n", [(2, 40), (100, 40), (1100, 1000)])
def test_matmul_far_scales(dt, m, n):
    """Scale bytes from one end to the other: products in and around fp32's range."""
    a, b = _q(m, 512, "e4m3", 6), _q(n, 512, "e4m3", 7)
    for i, s in enumerate((0, 1, 120, 220)):
        a.scales[:, i], b.scales[:, i] = s, 245 - s
    got = kge.matmul_quantized(a, b, dtype=dt)
    want, tol = _product(a, b, None, dt)
    _within(got, want, tol + (want.abs() + tol) * HALF[dt], "matmul")


def test_matmul_splits_only_as_far_as_the_workspace_goes():
    lib = kge.load()
    x, w = _q(130, 6000, "e4m3", 8), _q(140, 6000, "e4m3", 9)
    need = lib.kge_matmul_quantized_workspace_bytes(130, 140, 6000)
    assert need > 2 * 130 * 140 * 4
    want, tol = _product(x, w, None, F32)
    ws = torch.empty(need + 8, dtype=torch.uint8, device="cuda")
    for ptr, size in [(0, 0), (ws.data_ptr(), 100), (ws.data_ptr() + 8, need), (ws.data_ptr(), need // 2), (ws.data_ptr(), need)]:
        out = torch.full((130, 140), float("nan"), device="cuda")
        assert lib.kge_matmul_quantized(x.ref, None, 130, w.ref, 0, out.data_ptr(), 0, 140, ptr, size,
                                        torch.cuda.current_stream().cuda_stream) == 0
        _within(out, want, tol + (want.abs() + tol) * U)


# ---------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------
def _layer(table, w, ids, dy, drop1, drop2, ws=None):
    """One projection of scaled, dropped-out token embeddings with a residual, and its gradients, as a training step runs it."""
    V, d = table.shape
    x = kge.embed(table, ids, scale=4.0, dropout=drop1, dtype=BF16)
    xr, xc = kge.quantize(x, by="both")
    wr, wc = kge.quantize(w, by="both")
    y = kge.dropout(kge.matmul_quantized(xr, wr, ws=ws), drop2, residual=x)
    dz = kge.dropout(dy, drop2)
    zr, zc = kge.quantize(dz, fmt="e5m2", by="both")
    dw = kge.matmul_quantized(zc, xc, dtype=F32, ws=ws)
    dx = kge.matmul_quantized(zr, wc, ws=ws)
    dx = (dx.float() + dy.float()).to(BF16)
    return y, dw, kge.embed_bwd(dx, ids, V, scale=4.0, dropout=drop1, ws=ws)


def test_a_training_step_of_them_all():
    V, d, M = 40, 96, 150
    table, w, dy = _values((V, d), F32, 60, std=0.1), _values((d, d), F32, 61, std=0.1), _values((M, d), BF16, 62)
    ids = _ids(M, V, 63)
    d1, d2 = kge.Dropout(0.1, SEED, STEP, 1), kge.Dropout(0.25, SEED, STEP, 2)
    y, dw, dt = (t.double().cpu() for t in _layer(table.cuda(), w.cuda(), ids.cuda(), dy.cuda(), d1, d2))
    # the same step in 64 bits without any rounding
    f1, f2 = _factor(M, d, round(0.1 * 65536) / 65536, tag=1), _factor(M, d, 0.25, tag=2)
    live = ((ids >= 0) & (ids < V)).double().unsqueeze(1)
    at = ids.long().clamp(0, V - 1)
    x = table.double()[at] * 4 * f1 * live
    ry = (x @ w.double().t()) * f2 + x
    dz = dy.double() * f2
    rdw, rdx = dz.t() @ x, dz @ w.double() + dy.double()
    rdt = torch.zeros((V, d), dtype=torch.float64).index_add_(0, at, rdx * 4 * f1 * live)
    # an operand in e4m3 is off by 2^-4 of itself at most, in e5m2 by 2^-3 (plus the smallest codes' spacing, 2^-16 of the block's largest); a bf16
    # value by 2^-8: products of such operands, errors added up
    ax, aw, az = x.abs(), w.double().abs(), dz.abs()
    ey = ((2 ** -4 + 2 ** -4 + 2 ** -7 + 2 ** -8) * 1.01 * ((ax + ax.max() * 2 ** -15) @ (aw + aw.max() * 2 ** -15).t())) * f2 + 3 * 2 ** -8 * (ry.abs() + ax)
    assert bool(((y - ry).abs() <= ey + ey * 2 ** -7).all())
    ew = (2 ** -3 + 2 ** -4 + 2 ** -6) * 1.05 * ((az + az.max() * 2 ** -15).t() @ (ax + ax.max() * 2 ** -15))
    assert bool(((dw - rdw).abs() <= ew).all())
    ex = (2 ** -3 + 2 ** -4 + 2 ** -6) * 1.05 * ((az + az.max() * 2 ** -15) @ (aw + aw.max() * 2 ** -15)) + 3 * 2 ** -8 * (rdx.abs() + dy.double().abs())
    et = torch.zeros((V, d), dtype=torch.float64).index_add_(0, at, ex * 4 * f1 * live)
    assert bool(((dt - rdt).abs() <= et * 1.01).all())


def _graph_inputs(V, d, M, key):
    table, w, dy = _values((V, d), F32, key, std=0.1).cuda(), _values((d, d), F32, key + 1, std=0.1).cuda(), _values((M, d), BF16, key + 2).cuda()
    return table, w, _ids(M, V, key + 3).cuda(), dy


def _captured(step):
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                          # (the workspace's size, first launches)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step()
    return graph, out


@pytest.mark.parametrize("V,d,M", [(300, 96, 1100), (500, 64, 40_000)])
def test_the_step_in_a_graph_with_a_device_counter(V, d, M):
    """Captured once, replayed with the counter moving on: every replay equals the eager step of its number, with eager work between them."""
    args = _graph_inputs(V, d, M, 64)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    drops = [kge.Dropout(0.1, SEED, 5, t, step_counter=counter) for t in (1, 2)]
    eager = [_layer(*args, kge.Dropout(0.1, SEED, 5 + s, 1), kge.Dropout(0.1, SEED, 5 + s, 2)) for s in range(4)]
    ws = kge.Workspace()

    def step():
        out = _layer(*args, *drops, ws=ws)
        kge.step_counter_add(counter)
        return out
    graph, out = _captured(step)
    counter.zero_()
    for s in range(4):
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, eager[s]):
            assert torch.equal(got, want), s
        other = _layer(*args, kge.Dropout(0.1, SEED, 90, 1), kge.Dropout(0.1, SEED, 90, 2))   # eager work in between
        assert not torch.equal(other[0], out[0])


def test_two_graphs_and_eager_work_with_workspaces_of_their_own():
    cases = [_graph_inputs(300, 96, 1100, 80), _graph_inputs(900, 64, 36_000, 90)]
    d = kge.Dropout(0.2, SEED, 1, 1), kge.Dropout(0.3, SEED, 1, 2)
    want = [_layer(*c, *d) for c in cases]
    ws = [kge.Workspace() for _ in cases]
    graphs = [_captured(lambda c=c, w=w: _layer(*c, *d, ws=w)) for c, w in zip(cases, ws)]
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for k in order:
            graphs[k][0].replay()
        eager = _layer(*cases[1], *d)
        torch.cuda.synchronize()
        for k in (0, 1):
            for got, ref in zip(graphs[k][1], want[k]):
                assert torch.equal(got, ref)
        assert all(torch.equal(x, y) for x, y in zip(eager, want[1]))


def test_a_captured_call_without_a_workspace_of_its_own_is_refused():
    g, ids = _values((50, 64), F32, 95).cuda(), _ids(50, 20, 96).cuda()
    out = kge.embed_bwd(g, ids, 20)
    for ws in (None, kge.Workspace()):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            with pytest.raises(kge.KgeError, match="workspace"):
                kge.embed_bwd(g, ids, 20, out=out, ws=ws)
            out.add_(1)                                                 # (a graph needs a node)


def test_on_other_streams_at_once():
    """The same calls on three streams side by side, each with the scratch space that the library keeps for its stream."""
    table, ids = _values((100, 64), F32, 70).cuda(), _ids(40_000, 100, 71).cuda()
    g = _values((40_000, 64), F32, 72).cuda()
    q = kge.quantize(g, by="col")
    calls = [lambda s: kge.embed_bwd(g, ids, 100, stream=s), lambda s: kge.embed(table, ids, stream=s), lambda s: kge.quantize(g, stream=s).codes,
             lambda s: kge.matmul_quantized(q, q, dtype=F32, stream=s), lambda s: kge.dropout(g, kge.Dropout(0.5, 1), stream=s)]
    want = [c(None) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s in (*streams, None):
            got += [[c(s) for c in calls]]
    with torch.cuda.stream(streams[0]):
        got += [[c(None) for c in calls]]
    torch.cuda.synchronize()
    for outs in got:
        assert all(torch.equal(x, y) for x, y in zip(outs, want))


# ---------------------------------------------------------------------------------------------------------------
# places beyond 32 bits
# ---------------------------------------------------------------------------------------------------------------
def test_lookup_and_its_gradient_beyond_32_bits():
    n, d = 2_300_000, 1000                                              # 4.6 GB in bf16, 9.2 GB in fp32
    table = torch.zeros((n, d), dtype=BF16, device="cuda")
    rows = torch.tensor([0, 1, 2_147_483, 2_147_484, n - 1], dtype=torch.int32)
    v = _values((5, d), BF16, 100)
    table[rows.long().cuda()] = v.cuda()
    ids = rows[[4, 2, 0, 3, 1, 4]].cuda()
    assert torch.equal(kge.embed(table, ids).cpu(), v[[4, 2, 0, 3, 1, 4]])
    del table
    g = _values((6, d), F32, 101)
    for M in (6, 5000, 40_000):                                         # (one launch, three, and five)
        more = torch.full((M - 6,), -1, dtype=torch.int32, device="cuda")
        got = kge.embed_bwd(torch.cat([g.cuda(), torch.zeros((M - 6, d), device="cuda")]), torch.cat([ids, more]), n)
        want = torch.stack([g[2], g[4], g[1], g[3], g[0] + g[5]])
        assert torch.equal(got[rows.long().cuda()].cpu(), want)
        got[rows.long().cuda()] = 0
        assert not bool(got.any())
        del got


def test_dropout_and_quantisation_beyond_32_bits():
    rows, cols = 4_500_000, 1000
    x = torch.ones((rows, cols), dtype=BF16, device="cuda")
    d = kge.Dropout(0.25, SEED, STEP, TAG)
    q = kge.quantize(x)
    assert bool((q.codes.view(torch.int64).view(rows, 128)[:, :125] == q.codes.view(torch.int64)[0, 0]).all()) and bool((q.scales[:, :8] == 127 - 8).all())
    del q
    kge.dropout(x, d, out=x)
    for r in (0, 1, 4_294_967, 4_294_968, rows - 1):
        assert torch.equal(x[r:r + 1].cpu(), _factor(1, cols, 0.25, row0=r).to(BF16))


def _random_codes(rows, cols, key):
    """Codes that stand for +-1, +-1.5, +-2, +-3 (scale 1): sums are whole halves, exact in fp32 whatever their order."""
    g = torch.Generator(device="cuda").manual_seed(key)
    pick = torch.tensor([0x38, 0x3C, 0x40, 0x44, 0xB8, 0xBC, 0xC0, 0xC4], dtype=torch.uint8, device="cuda")
    codes = torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
    for part in codes.split(1 << 16):
        part.copy_(pick[torch.randint(0, 8, part.shape, generator=g, device="cuda")])
    return kge.Quantized(codes, torch.full((rows, -(-cols // 512) * 4), 127, dtype=torch.uint8, device="cuda"), cols)


def _values_of(q, rows):
    return _decode(q.codes[rows].cpu(), "e4m3")


def test_product_of_rows_beyond_32_bits():
    """A gathered table of 4.6 GB (64-bit addresses in every kernel that gathers), and offsets between 2 and 4 GB in the kernel with 32-bit ones."""
    table = _random_codes(4_500_000, 1024, 1)
    b = _random_codes(300, 1024, 2)
    at = torch.tensor([0, 4_194_303, 4_194_304, 4_499_999, 2_097_152])
    for m in (5, 200, 3000):
        rows = at[torch.arange(m) % 5].to(torch.int32).cuda()
        got = kge.matmul_quantized(table, b, rows=rows, dtype=F32).double().cpu()
        want = _values_of(table, at.cuda()) @ _values_of(b, torch.arange(300, device="cuda")).t()
        assert torch.equal(got, want[torch.arange(m) % 5])
    near = kge.Quantized(table.codes[:4_100_000], table.scales[:4_100_000], 1024)       # 4.198 GB: just below 2^32
    rows = torch.arange(4_100_000 - 70_000, 4_100_000, dtype=torch.int32, device="cuda")
    for dt in (F32, BF16):
        got = kge.matmul_quantized(near, b, rows=rows, dtype=dt)
        some = torch.tensor([0, 1, 255, 256, 33_333, 69_999])
        want = _values_of(near, rows[some.cuda()].long()) @ _values_of(b, torch.arange(300, device="cuda")).t()
        assert torch.equal(got[some.cuda()].double().cpu(), want.to(dt).double())


def test_product_of_scales_beyond_32_bits():
    """Scales with gaps, 5.2 GB from the first to the last, of a matrix whose codes are small."""
    a, b = _random_codes(5000, 128, 3), _random_codes(700, 128, 4)
    far = torch.zeros((5000, 1 << 20), dtype=torch.uint8, device="cuda")
    far[:, 0] = 127 + (torch.arange(5000, device="cuda") % 5).to(torch.uint8)
    a = kge.Quantized(a.codes, far[:, :4], 128)
    rows = torch.arange(20_000, dtype=torch.int32) % 5000
    some = torch.tensor([0, 1, 4095, 4096, 4999, 19_998])
    want = _values_of(a, rows[some].long().cuda()) * 2.0 ** (rows[some] % 5).double().unsqueeze(1) @ _values_of(b, torch.arange(700, device="cuda")).t()
    for m in (100, 20_000):
        got = kge.matmul_quantized(a, b, rows=rows[:m].cuda(), dtype=F32)
        ok = some < m
        assert torch.equal(got[some[ok].cuda()].double().cpu(), want[ok])


def test_the_binding_refuses():
    x = torch.zeros((4, 64), device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    d = kge.Dropout(0.5, 1)
    q = kge.quantize(x)
    for call in [lambda: kge.embed(x.cpu(), ids), lambda: kge.embed(x, ids.long()), lambda: kge.embed(x.half(), ids), lambda: kge.embed(x.t(), ids),
                 lambda: kge.embed(x, ids, out=torch.empty((4, 63), device="cuda")), lambda: kge.embed_bwd(x, ids[:3], 9),
                 lambda: kge.embed_bwd(x, ids, 9, accumulate=True), lambda: kge.dropout(x, d, residual=x[:3]), lambda: kge.dropout(x, d, residual=x.bfloat16()),
                 lambda: kge.dropout(x, d, out=torch.empty((4, 64), dtype=torch.bfloat16, device="cuda")), lambda: kge.dropout(x, kge.Dropout(1.0, 1)),
                 lambda: kge.quantize(x, by="rows"), lambda: kge.Quantized(q.codes[:, :64], q.scales, 64), lambda: kge.Quantized(q.codes, q.scales[:, :1], 64),
                 lambda: kge.Quantized(q.codes, q.scales, 200), lambda: kge.matmul_quantized(q, kge.quantize(torch.zeros((4, 200), device="cuda"))),
                 lambda: kge.matmul_quantized(q, q, accumulate=True), lambda: kge.matmul_quantized(q, q, rows=ids.long()),
                 lambda: kge.matmul_quantized(q, q, out=torch.empty((4, 5), device="cuda")), lambda: kge.dropout(x.expand(4, 64)[:, :1].expand(4, 64), d),
                 lambda: kge.quantize(x, fmt="e3m4"), lambda: kge.quantize(x, fmt="e5m2", out=q), lambda: kge.quantize(x, by="both", out=q),
                 lambda: kge.Quantized(q.codes, q.scales, 64, "fp8")]:
        with pytest.raises(kge.KgeError):
            call()
