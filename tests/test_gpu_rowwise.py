"""Matrices in 8-bit integers with a scale per row: the quantiser and the product, bit for bit against fp32 arithmetic on the CPU."""
import numpy as np
import pytest
import torch

import paper_2211_12281_amd as kge

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def _rng(*key):
    return np.random.default_rng([int(k) for k in key])


def _values(shape, dtype, *key, std=1.0):
    return (torch.from_numpy(_rng(*key).normal(size=shape)) * std).to(dtype)


def _padded(t, pad):
    if pad == 0:
        return t.cuda()
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, pad // 2:pad // 2 + t.shape[1]] = t.cuda()
    return wide[:, pad // 2:pad // 2 + t.shape[1]]


# ---------------------------------------------------------------------------------------------------------------
# quantisation
# ---------------------------------------------------------------------------------------------------------------
def _quantized(x):
    """(codes int64 [rows, padded], scales) in numpy's fp32, each operation rounded once."""
    x = x.float().numpy()
    rows, cols = x.shape
    amax = np.abs(x).max(axis=1) if cols else np.zeros(rows, np.float32)
    ok = np.isfinite(amax)
    a = np.maximum(np.where(ok, amax, np.float32(1)), np.float32(2.0 ** -100)).astype(np.float32)
    inv, scale = np.float32(127) / a, a / np.float32(127)
    codes = np.zeros((rows, -(-cols // 128) * 128), dtype=np.int64)
    with np.errstate(invalid="ignore", over="ignore"):
        q = np.rint(x * inv[:, None])
    codes[:, :cols] = np.where(ok[:, None], q, 0).astype(np.int64)
    return torch.from_numpy(codes), torch.from_numpy(np.where(ok, scale, np.float32("nan")).astype(np.float32))


def _same(q, x):
    codes, scales = _quantized(x)
    assert (q.rows, q.cols) == tuple(x.shape)
    got = q.codes[:, :codes.shape[1]].cpu().long()
    assert torch.equal(got, codes), (got != codes).nonzero()[:3]
    assert torch.equal(torch.nan_to_num(q.scales.cpu(), nan=-1.0), torch.nan_to_num(scales, nan=-1.0))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 1), (5, 128, 0), (130, 129, 3), (257, 300, 1), (2, 513, 0), (7, 1025, 1), (3, 2049, 0), (2, 4097, 1), (3, 8193, 0),
                                           (2, 32_769, 1), (1, 131_071, 0), (700, 64, 0), (128, 128, 0), (256, 31, 1), (511, 33, 0), (512, 200, 1), (513, 200, 0)])
@pytest.mark.parametrize("by", ["row", "col", "both"])
def test_quantize(dt, rows, cols, pad, by):
    x = _values((rows, cols), dt, 1, rows, cols) * torch.from_numpy(_rng(2, rows).uniform(1e-3, 1e3, size=(rows, 1))).to(dt)
    q = kge.quantize_rowwise(_padded(x, pad), by=by)
    for layout, t in zip(q if by == "both" else (q,), (x, x.t()) if by == "both" else ((x,) if by == "row" else (x.t(),))):
        _same(layout, t)


@pytest.mark.parametrize("rows,cols", [(40_000, 96), (131_071, 3), (3, 131_071)])
def test_quantize_long_columns(rows, cols):
    x = _values((rows, cols), BF16, 3, rows)
    _same(kge.quantize_rowwise(x.cuda(), by="col"), x.t())


def test_quantize_extremes():
    """Rows of zeros, of the smallest and largest numbers, of halves that round to even, and of what is not finite."""
    x = torch.zeros((12, 200))
    x[1, 3] = 2.0 ** -149
    x[2] = 2.0 ** -101 * torch.linspace(-1, 1, 200)
    x[3] = 2.0 ** -100 * torch.linspace(-1, 1, 200)
    x[4] = torch.finfo(F32).max * torch.linspace(-1, 1, 200)
    x[5] = torch.arange(200) - 99.5
    x[5, 0] = 127.0
    x[6, 7], x[7, 199], x[8, 0] = float("nan"), float("inf"), float("-inf")
    x[6, 8:], x[8, 100:] = 1.0, float("inf")
    x[9] = -0.0
    x[10] = -3.0
    x[11, 0], x[11, 1] = 1.0, 2.0 ** -20
    for by in ("row", "both"):
        q = kge.quantize_rowwise(x.cuda(), by=by)
        _same(q[0] if by == "both" else q, x)
        if by == "both":
            _same(q[1], x.t())
    q = kge.quantize_rowwise(x[:, :1].contiguous().cuda().expand(12, 1), by="col")
    _same(q, x[:, :1].t())


@pytest.mark.parametrize("by", ["row", "col"])
def test_quantize_writes_its_rows_alone(by):
    x = _values((37, 90), F32, 4)
    rows = 37 if by == "row" else 90
    wide = torch.full((rows + 2, 256), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((rows + 2,), 5.0, device="cuda")
    out = kge.Rowwise(wide[1:-1, :240], scales[1:-1], 90 if by == "row" else 37)
    assert out.struct.ld == 256
    assert kge.quantize_rowwise(x.cuda(), by=by, out=out) is out
    _same(out, x if by == "row" else x.t())
    assert bool((wide[0] == 77).all()) and bool((wide[-1] == 77).all()) and bool((wide[:, 128:] == 77).all()) and scales[0] == 5 and scales[-1] == 5


def test_quantize_of_nothing():
    q = kge.quantize_rowwise(torch.empty((0, 9), device="cuda"))
    assert q.rows == 0
    q = kge.quantize_rowwise(torch.empty((0, 9), device="cuda"), by="col")
    y = kge.matmul_rowwise(q, q, dtype=F32)
    assert y.shape == (9, 9) and not bool(y.any())
    q = kge.quantize_rowwise(torch.empty((5, 0), device="cuda"))
    assert not bool(kge.matmul_rowwise(q, q, dtype=F32).any())


@pytest.mark.parametrize("rows", [0, 5, 600])
def test_quantize_of_no_columns_both_ways(rows):
    q, t = kge.quantize_rowwise(torch.empty((rows, 0), device="cuda"), by="both")
    assert (q.rows, q.cols, t.rows, t.cols) == (rows, 0, 0, rows)
    _same(q, torch.empty((rows, 0)))
    y = kge.matmul_rowwise(q, q, dtype=F32)
    assert y.shape == (rows, rows) and not bool(y.any())
    assert kge.matmul_rowwise(t, t).shape == (0, 0)


# ---------------------------------------------------------------------------------------------------------------
# product
# ---------------------------------------------------------------------------------------------------------------
def _matrix(rows, cols, *key, top=127):
    g = _rng(*key, rows, cols)
    codes = np.zeros((rows, -(-cols // 128) * 128), dtype=np.int8)
    codes[:, :cols] = g.integers(-top, top + 1, size=(rows, cols))
    return torch.from_numpy(codes), torch.from_numpy(g.uniform(1e-3, 1e-1, size=rows).astype(np.float32))


def _cuda(q, cols):
    return kge.Rowwise(q[0].cuda(), q[1].cuda(), cols)


def _product(a, b, rows=None):
    """fp32 [m, n]: exact sums, then the roundings of the call; rows outside give zeros"""
    codes, scales = a
    if rows is not None:
        live = (rows >= 0) & (rows < codes.shape[0])
        at = torch.where(live, rows, torch.zeros_like(rows)).long()
        codes, scales = codes[at], scales[at]
    sums = codes.double() @ b[0].double().t()                    # (whole numbers below 2^53)
    y = sums.float() * scales.unsqueeze(1) * b[1]
    return y if rows is None else torch.where(live.unsqueeze(1), y, torch.zeros(()))


def _equal(got, want):
    got = got.cpu()
    assert got.dtype == want.dtype and got.shape == want.shape
    assert torch.equal(got, want), (got != want).nonzero()[:3]


SHAPES = [(1, 1, 1), (1, 30, 100), (7, 16, 128), (16, 300, 257), (17, 33, 1000), (65, 129, 300), (130, 128, 700), (200, 97, 4200), (300, 700, 900), (257, 256, 130),
          (64, 4096, 2000), (1, 5000, 4096), (1030, 1029, 200), (768, 640, 9000)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_matmul(dt, m, n, k):
    a, b = _matrix(m, k, 5), _matrix(n, k, 6)
    _equal(kge.matmul_rowwise(_cuda(a, k), _cuda(b, k), dtype=dt), _product(a, b).to(dt))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(4100, 4090, 300), (4096, 4096, 128), (65_600, 300, 200), (300, 60_000, 400), (3500, 3600, 1500)])
def test_matmul_large_tiles(dt, m, n, k):
    """Products of many tiles, on the GPU's own 64-bit sums."""
    a, b = _matrix(m, k, 7), _matrix(n, k, 8)
    want = ((a[0].cuda().double() @ b[0].cuda().double().t()).float() * a[1].cuda().unsqueeze(1) * b[1].cuda()).to(dt)
    got = kge.matmul_rowwise(_cuda(a, k), _cuda(b, k), dtype=dt)
    assert torch.equal(got, want), (got != want).nonzero()[:3]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m,n,k,pad", [(5, 30, 300, 1), (90, 131, 260, 3), (200, 96, 4200, 2), (1, 7, 128, 0), (1030, 1029, 200, 3), (300, 1700, 1300, 1), (4200, 4100, 140, 1)])
def test_matmul_gathered_accumulated_strided(dt, m, n, k, pad):
    table, b = _matrix(501, k, 9), _matrix(n, k, 10)
    g = _rng(11, m)
    rows = torch.from_numpy(g.integers(0, 501, size=m).astype(np.int32))
    rows[g.integers(0, m, size=max(1, m // 20))] = -1
    rows[0] = 501 if m > 1 else 0
    rows[m // 2] = 500
    old = _values((m, n), dt, 12, m)
    out = _padded(old, pad)
    wide = torch.full((501, table[0].shape[1] + 48), 99, dtype=torch.int8, device="cuda")
    wide[:, :table[0].shape[1]] = table[0].cuda()
    a = kge.Rowwise(wide[:, :-48], table[1].cuda(), k)
    got = kge.matmul_rowwise(a, _cuda(b, k), rows=rows.cuda(), out=out, accumulate=True)
    assert got is out
    y = _product(table, b, rows).double()
    want = y + old.double()
    # the product's last rounding and the addition's (or both at once), then the output's
    tol = U * (y.abs() + want.abs()) + (2.0 ** -8 if dt == BF16 else 0.0) * want.abs() * (1 + U)
    assert bool(((got.double().cpu() - want).abs() <= tol).all())
    if pad > 1:
        assert bool(torch.isnan(out._base[:, 0]).all()) and bool(torch.isnan(out._base[:, -1]).all())
    _equal(kge.matmul_rowwise(a, _cuda(b, k), rows=rows.cuda(), dtype=dt), _product(table, b, rows).to(dt))


@pytest.mark.parametrize("m,n,k", [(2100, 2101, 100), (2250, 2000, 1000), (8200, 500, 640), (20_000, 256, 129), (9000, 511, 260)])
def test_matmul_of_wide_tiles(m, n, k):
    """Tiles of 128 x 256: more than a compute unit has of 128 x 128; gathered rows, and added to what is there."""
    a, b = _matrix(m, k, 19), _matrix(n, k, 20)
    rows = torch.from_numpy(_rng(21, k).integers(-1, m + 1, size=m).astype(np.int32)).cuda()
    qa, qb = _cuda(a, k), _cuda(b, k)
    want = (a[0].cuda().double() @ b[0].cuda().double().t()).float() * a[1].cuda().unsqueeze(1) * b[1].cuda()
    for dt in (F32, BF16):
        got = kge.matmul_rowwise(qa, qb, dtype=dt)
        assert torch.equal(got, want.to(dt)), (got != want.to(dt)).nonzero()[:3]
    live = (rows >= 0) & (rows < m)
    taken = torch.where(live.unsqueeze(1), want[rows.clamp(0, m - 1).long()], torch.zeros((), device="cuda"))
    got = kge.matmul_rowwise(qa, qb, rows=rows, dtype=BF16)
    assert torch.equal(got, taken.to(BF16))
    out = torch.full((m, n), 0.0, device="cuda")
    kge.matmul_rowwise(qa, qb, rows=rows, dtype=F32, out=out, accumulate=True)
    assert torch.equal(out, taken)


@pytest.mark.parametrize("k", [1921, 2048, 2100, 2300, 2432, 2433, 3900, 4096, 6200, 20_001])
def test_matmul_of_a_workgroup_per_compute_unit(k):
    """Tiles that have a compute unit each, contractions of every length in blocks modulo the ring, whole and split; gathered rows too."""
    m, n = 700, 900
    a, b = _matrix(m, k, 16), _matrix(n, k, 17)
    rows = torch.from_numpy(_rng(18, k).integers(-1, m + 1, size=1300).astype(np.int32))
    qa, qb = _cuda(a, k), _cuda(b, k)
    sums = a[0].cuda().double() @ b[0].cuda().double().t()
    want = (sums.float() * a[1].cuda().unsqueeze(1) * b[1].cuda()).cpu()
    got = kge.matmul_rowwise(qa, qb, dtype=F32)
    _equal(got, want)
    _equal(kge.matmul_rowwise(qa, qb, dtype=BF16), want.to(BF16))
    live = (rows >= 0) & (rows < m)
    taken = torch.where(live.unsqueeze(1), want[rows.clamp(0, m - 1).long()], torch.zeros(()))
    _equal(kge.matmul_rowwise(qa, qb, rows=rows.cuda(), dtype=F32), taken)


@pytest.mark.parametrize("m,n", [(3, 20), (200, 130), (2100, 2000)])
def test_sums_reach_the_end_of_32_bits(m, n):
    """The longest contraction of the largest codes."""
    k = 131_071
    a = torch.zeros((m, 131_072), dtype=torch.int8, device="cuda")
    b = torch.zeros((n, 131_072), dtype=torch.int8, device="cuda")
    a[:, :k], b[:, :k] = 127, -127
    b[1, :k] = 127
    one = lambda r: torch.ones(r, device="cuda")                  # noqa: E731
    got = kge.matmul_rowwise(kge.Rowwise(a, one(m), k), kge.Rowwise(b, one(n), k), dtype=F32)
    want = torch.full((m, n), float(np.float32(-127 * 127 * k)))
    want[:, 1] = float(np.float32(127 * 127 * k))
    _equal(got, want)


@pytest.mark.parametrize("m,n", [(3, 40), (100, 40), (1100, 1000)])
def test_a_nan_scale_stays_in_its_row(m, n):
    a, b = _matrix(m, 300, 13), _matrix(n, 300, 14)
    a[1][1], b[1][2] = float("nan"), float("inf")
    b[0][2] = 0
    got = kge.matmul_rowwise(_cuda(a, 300), _cuda(b, 300), dtype=F32).cpu()
    assert bool(torch.isnan(got[1]).all()) and bool(torch.isnan(got[:, 2]).all())
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[1], keep[:, 2] = False, False
    assert torch.equal(got[keep], _product(a, b)[keep])


def test_matmul_gathers_nothing_from_an_empty_table():
    q = kge.Rowwise.empty(0, 70)
    got = kge.matmul_rowwise(q, _cuda(_matrix(9, 70, 15), 70), rows=torch.tensor([0, -1, 3], dtype=torch.int32, device="cuda"))
    assert got.shape == (3, 9) and not bool(got.any())


def test_splits_do_not_change_the_result():
    m, n, k = 200, 700, 9000                                      # (a product that is split)
    a, b = _matrix(m, k, 16), _matrix(n, k, 17)
    want = _product(a, b)
    lib, da, db = kge.load(), _cuda(a, k), _cuda(b, k)
    need = lib.kge_matmul_rowwise_workspace_bytes(m, n, k)
    assert need > 256 + 4 * m * n
    for size in (need, 3 * 4 * m * n + 300, 256, 0):
        out, ws = torch.full((m, n), float("nan"), device="cuda"), torch.empty(max(size, 1) + 8, dtype=torch.uint8, device="cuda")
        assert lib.kge_matmul_rowwise(da.ref, None, m, db.ref, 0, out.data_ptr(), 0, n, ws.data_ptr() + 8 if size else None, size, None) == 0
        torch.cuda.synchronize()
        _equal(out, want)


def test_product_of_rows_beyond_32_bits():
    rows, k = 5_600_000, 768                                      # codes of 4.3 GB
    codes = torch.zeros((rows, k), dtype=torch.int8, device="cuda")
    b = _matrix(300, k, 18)
    last = _matrix(400, k, 19)
    codes[-400:] = last[0].cuda()
    scales = torch.ones(rows, device="cuda")
    scales[-400:] = last[1].cuda()
    a = kge.Rowwise(codes, scales, k)
    for m in (5, 400):
        ids = torch.arange(rows - m, rows, dtype=torch.int32)
        _equal(kge.matmul_rowwise(a, _cuda(b, k), rows=ids.cuda(), dtype=F32), _product((last[0][-m:], last[1][-m:]), b))
    got = kge.matmul_rowwise(a, _cuda((b[0][:8], b[1][:8]), k), dtype=BF16)
    _equal(got[-400:], _product(last, (b[0][:8], b[1][:8])).to(BF16))
    assert not bool(got[:-400].any())


def test_captured_calls_are_replayed():
    x, w = _values((1500, 520), BF16, 20).cuda(), _values((64, 520), BF16, 21).cuda()
    wq = kge.quantize_rowwise(w, by="both")

    def layer(ws):
        qr, qc = kge.quantize_rowwise(x, by="both", ws=ws[0])
        y = kge.matmul_rowwise(qr, wq[0], dtype=F32, ws=ws[1])
        return [qr.codes, qr.scales, qc.codes, qc.scales, y, kge.matmul_rowwise(qc, kge.quantize_rowwise(y, by="col", ws=ws[2]), dtype=F32, ws=ws[3])]
    spaces = [kge.Workspace() for _ in range(4)]
    for s in spaces:
        s.get(64 << 20)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(spaces)
    for i in range(4):
        x.copy_(_values(x.shape, BF16, 22, i))
        want = layer([None] * 4)
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i


def test_the_binding_refuses():
    x = torch.zeros((4, 8), device="cuda")
    q = kge.quantize_rowwise(x)
    for bad in [lambda: kge.quantize_rowwise(x, by="diagonal"), lambda: kge.quantize_rowwise(x.cpu()), lambda: kge.quantize_rowwise(x.half()),
                lambda: kge.quantize_rowwise(x, out=kge.Rowwise.empty(5, 8)), lambda: kge.quantize_rowwise(x, by="both", out=q),
                lambda: kge.quantize_rowwise(torch.zeros((1, 131_072), device="cuda")), lambda: kge.quantize_rowwise(torch.zeros((131_072, 1), device="cuda"), by="col"),
                lambda: kge.Rowwise(q.codes[:, :100], q.scales, 8), lambda: kge.Rowwise(q.codes, q.scales[:3], 8), lambda: kge.Rowwise(q.codes.to(torch.uint8), q.scales, 8),
                lambda: kge.Rowwise(q.codes, q.scales.cpu(), 8), lambda: kge.matmul_rowwise(q, kge.Rowwise.empty(3, 9)), lambda: kge.matmul_rowwise(q, q, accumulate=True),
                lambda: kge.matmul_rowwise(q, q, dtype=torch.float16), lambda: kge.matmul_rowwise(q, q, rows=torch.zeros(3, device="cuda")),
                lambda: kge.matmul_rowwise(q, q, out=x)]:
        with pytest.raises(kge.KgeError):
            bad()
    with pytest.raises(kge.KgeError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            kge.quantize_rowwise(torch.zeros((600, 8), device="cuda"), by="col")
    torch.cuda.synchronize()
