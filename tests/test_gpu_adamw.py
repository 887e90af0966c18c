"""AdamW over many dense tensors against plain arithmetic on the CPU: moments bit for bit (their operations are rounded one by one), parameters to the
roundings of the update."""
import math

import numpy as np
import pytest
import torch

import paper_2211_12281_amd as kge

pytestmark = pytest.mark.gpu
F, F32, BF16 = np.float32, torch.float32, torch.bfloat16
U = 2.0 ** -24
CFG = dict(lr=F(1e-3), b1=F(0.9), b2=F(0.999), eps=F(1e-8))


def _rng(*key):
    return np.random.default_rng([int(k) for k in key])


def _philox(n, tensor, step, seed, tag):
    """uint32 [n]: word i % 4 of the block of counter (i / 4, tensor, step, tag), on Python integers."""
    out = []
    for g in range(-(-n // 4)):
        c, k = [g, tensor, step & 0xFFFFFFFF, tag], [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [p1 >> 32 ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, p0 >> 32 ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        out += c
    return np.array(out[:n], dtype=np.uint64)


def _grid(fmt):
    """Values of the codes 0..top of a format."""
    bits, emin, top = (3, -6, 0x7e) if fmt == "e4m3" else (2, -14, 0x7b)
    return np.array([(c % (1 << bits) + ((1 << bits) if c >> bits else 0)) * 2.0 ** (max(c >> bits, 1) - 1 + emin - bits) for c in range(top + 1)])


GRID = {f: _grid(f) for f in ("e4m3", "e5m2")}


def _decode(codes, scales, n, fmt):
    c = codes.cpu().numpy()[:n].astype(np.int64)
    mag = c & 0x7f
    v = np.where(mag < len(GRID[fmt]), GRID[fmt][np.minimum(mag, len(GRID[fmt]) - 1)], np.nan)
    if fmt == "e5m2":
        v = np.where(mag == 0x7c, np.inf, v)
    s = scales.cpu().numpy().astype(np.float64)[np.arange(n) // 128]
    return np.where(c >> 7, -v, v) * 2.0 ** (s - 127)


def _byte(x, fmt):
    """Scale byte of a block, from its finite elements."""
    a = np.abs(x[np.isfinite(x)].astype(np.float64))
    a = a.max() if a.size else 0.0
    if a == 0:
        return 0
    e = math.frexp(a)[1] - 1 - (8 if fmt == "e4m3" else 15)
    e += a > GRID[fmt][-1] * 2.0 ** e
    return min(max(e + 127, 0), 254)


def _check_codes(codes, scales, x, fmt, u):
    """Codes of the fp32 values x: the neighbour below, or above where the fraction between them + u reaches one (within 2^-19 of that either: the sum is rounded)."""
    n, nb = x.size, -(-x.size // 128)
    s = scales.cpu().numpy()
    for i in range(nb):
        assert s[i] == _byte(x[128 * i:128 * (i + 1)], fmt), (i, s[i])
    got = codes.cpu().numpy()
    assert not got[n:].any()
    fine = np.isfinite(x)
    mag = got[:n].astype(np.int64) & 0x7f
    t = np.abs(np.where(fine, x, 0).astype(np.float64)) * 2.0 ** (127.0 - s[np.arange(n) // 128])
    grid = GRID[fmt]
    lo = np.searchsorted(grid, t, side="right") - 1
    hi = np.minimum(lo + 1, len(grid) - 1)
    frac = np.where(hi > lo, (t - grid[lo]) / np.where(hi > lo, grid[hi] - grid[lo], 1), 0.0)
    up = frac + u >= 1
    want = np.where(up, hi, lo)
    either = np.abs(frac + u - 1) < 2.0 ** -19
    if fmt == "e5m2":
        want = np.where((t > 0) & (want == 0), 1, want)
    ok = (mag == want) | (either & ((mag == lo) | (mag == hi)))
    assert ok[fine].all(), (np.nonzero(~ok & fine)[0][:3], mag[~ok & fine][:3], want[~ok & fine][:3])
    assert (np.signbit(x[fine]) == (got[:n][fine] >> 7).astype(bool))[mag[fine] > 0].all()
    bad = np.where(np.isinf(x), 0x7c, 0x7f) if fmt == "e5m2" else np.full(n, 0x7f)
    assert (mag[~fine] == bad[~fine]).all()


def _moments(m, v, g):
    """fp32, each operation rounded"""
    with np.errstate(over="ignore", invalid="ignore"):
        return m * CFG["b1"] + g * (F(1) - CFG["b1"]), v * CFG["b2"] + (g * g) * (F(1) - CFG["b2"])


def _check_params(got, p, m, v, wd, step):
    """Parameters from the new moments (fp32 values).  The update is c1 m lr / (sqrt(c2 v) + eps): c1, m c1, lr, the quotient and eps's sum a rounding each, c2 and v c2
    half of one behind the root, the root one; with 8-bit moments root and reciprocal are good to an ulp, two roundings each, and there is a product more: ten.
    Two roundings of the decay and one of the sum, relative to what is added."""
    p, m, v = (t.astype(np.float64) for t in (p, m, v))
    b1, b2, lr, eps = (float(CFG[k]) for k in ("b1", "b2", "lr", "eps"))
    with np.errstate(invalid="ignore"):
        upd = lr * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    want = p * (1 - lr * float(F(wd))) - upd
    tol = 10 * U * np.abs(upd) + 3 * U * (np.abs(p) + np.abs(want))
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine)
    assert (np.abs(got.astype(np.float64) - want) <= tol)[fine].all()


def _tensor(n, bits, gdt, shadow, key, off=0):
    """(param, grad, state, shadow) on the GPU, from an odd place of a larger buffer each, and the moments' values"""
    g = _rng(key, n)
    at = lambda a, dt: torch.cat([torch.zeros(off, dtype=dt), torch.from_numpy(a).to(dt), torch.full((3,), 7.0).to(dt)]).cuda()[off:off + n]     # noqa: E731
    p = at((g.normal(size=n) * 0.1).astype(F), F32)
    grad = at((g.normal(size=n) * 10.0 ** g.uniform(-6, -1, size=n)).astype(F), gdt)
    m, v = (g.normal(size=n) * 1e-3).astype(F), (g.normal(size=n) ** 2 * 1e-6).astype(F)
    if bits == 32:
        st = kge.AdamWState(at(m, F32), at(v, F32))
    else:
        st = kge.AdamWState.zeros(n, 8)
        nb = -(-n // 128)
        st.m[:n] = torch.from_numpy(g.integers(0, 0x7f, size=n).astype(np.uint8) | (g.integers(0, 2, size=n) << 7).astype(np.uint8)).cuda()
        st.v[:n] = torch.from_numpy(g.integers(0, 0x7c, size=n).astype(np.uint8)).cuda()
        st.m_scales[:nb] = torch.from_numpy(g.integers(100, 115, size=nb).astype(np.uint8)).cuda()
        st.v_scales[:nb] = torch.from_numpy(g.integers(80, 100, size=nb).astype(np.uint8)).cuda()
        m, v = _decode(st.m, st.m_scales, n, "e4m3").astype(F), _decode(st.v, st.v_scales, n, "e5m2").astype(F)
    return p, grad, st, (at(np.zeros(n), BF16) if shadow else None), m, v


def _run(sizes, bits, gdt, shadow, step=3, off=0, key=0, wd=0.01, **kw):
    ts = [_tensor(n, b, gdt, shadow, key + i, off) for i, (n, b) in enumerate(zip(sizes, bits))]
    before = [t[0].cpu().numpy().copy() for t in ts]
    opt = kge.AdamW([t[0] for t in ts], [t[2] for t in ts], shadows=[t[3] for t in ts], weight_decay=[wd * (i % 2) for i in range(len(ts))], seed=0xABCDEF0123456789, tag=9)
    opt.step([t[1] for t in ts], float(CFG["lr"]), step, eps=float(CFG["eps"]), **kw)
    return ts, before


def _check(ts, before, bits, step, wd=0.01, scale=None):
    for i, ((p, grad, st, sh, m, v), old, b) in enumerate(zip(ts, before, bits)):
        n = p.numel()
        g = grad.float().cpu().numpy()
        m, v = _moments(m, v, g if scale is None else g * F(scale))
        _check_params(p.cpu().numpy(), old, m, v, wd * (i % 2), step)
        if sh is not None:
            assert torch.equal(sh.cpu(), p.cpu().to(BF16))
        if b == 32:
            assert np.array_equal(st.m.cpu().numpy(), m) and np.array_equal(st.v.cpu().numpy(), v)
        else:
            w = _philox(n, i, step, 0xABCDEF0123456789, 9)
            _check_codes(st.m, st.m_scales, m, "e4m3", (w & 0xFFFF) / 65536)
            _check_codes(st.v, st.v_scales, v, "e5m2", (w >> 16) / 65536)
        for t in (p, grad, sh) + ((st.m, st.v) if b == 32 else ()):
            if t is not None and n and t._base is not None:
                assert bool((t._base[-3:] == 7).all())            # what lies behind a tensor stays


SIZES = [1, 3, 127, 128, 129, 2047, 2048, 2049, 5001]


@pytest.mark.parametrize("gdt", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("off", [0, 1])
def test_one_tensor(n, bits, gdt, off):
    ts, before = _run([n], [bits], gdt, off == 0, off=off, key=n)
    _check(ts, before, [bits], 3)


@pytest.mark.parametrize("shadow", [False, True])
def test_many_tensors_of_both_kinds(shadow):
    """More tensors than a launch takes, empty ones among them."""
    g = _rng(5)
    sizes = [int(n) for n in g.choice([0, 1, 5, 130, 700, 2500], size=97)]
    bits = [int(b) for b in g.choice([8, 32], size=97)]
    ts, before = _run(sizes, bits, BF16, shadow, key=50)
    _check(ts, before, bits, 3)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_times_a_number_on_the_device(bits):
    s = torch.tensor([0.37], device="cuda")
    ts, before = _run([1000, 77], [bits] * 2, F32, True, key=60, grad_scale=s)
    _check(ts, before, [bits] * 2, 3, scale=float(s.cpu()))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_from_a_counter_is_the_same_step(bits):
    a, _ = _run([900, 300], [bits] * 2, F32, True, step=12, key=70)
    b, before = _run([900, 300], [bits] * 2, F32, True, step=2, key=70, step_counter=torch.tensor([10], device="cuda"))
    for x, y in zip(a, b):
        for s, t in ((x[0], y[0]), (x[3], y[3]), (x[2].m, y[2].m), (x[2].v, y[2].v)):
            assert torch.equal(s, t)
    _check(b, before, [bits] * 2, 12)


@pytest.mark.parametrize("bits", [32, 8])
def test_what_is_not_finite_stays_with_its_element(bits):
    n = 400
    p, grad, st, sh, m, v = _tensor(n, bits, F32, True, 80)
    grad[5], grad[130], grad[131], grad[399] = float("nan"), float("inf"), float("-inf"), 3e38
    old = p.cpu().numpy().copy()
    kge.AdamW([p], [st], shadows=[sh], weight_decay=0.0, seed=0xABCDEF0123456789, tag=9).step([grad], float(CFG["lr"]), 3, eps=float(CFG["eps"]))
    got = p.cpu().numpy()
    assert np.isfinite(np.delete(got, [5, 130, 131, 399])).all() and np.isnan(got[[5, 130, 131]]).all()
    m, v = _moments(m, v, grad.cpu().numpy())
    if bits == 8:
        w = _philox(n, 0, 3, 0xABCDEF0123456789, 9)
        _check_codes(st.m, st.m_scales, m, "e4m3", (w & 0xFFFF) / 65536)
        _check_codes(st.v, st.v_scales, v, "e5m2", (w >> 16) / 65536)
    else:
        assert np.array_equal(st.m.cpu().numpy(), m, equal_nan=True) and np.array_equal(st.v.cpu().numpy(), v, equal_nan=True)
    assert old.shape == got.shape


def test_8_bit_moments_of_zeros_and_of_every_binade():
    """Zeros stay zeros, a positive second moment never becomes one, and blocks from the smallest to the largest numbers have their scales."""
    n = 128 * 60
    p, st = torch.ones(n, device="cuda"), kge.AdamWState.zeros(n, 8)
    mag = np.repeat(2.0 ** np.linspace(-70, 62, 60), 128) * _rng(81).uniform(0.0, 1.0, size=n) ** 12
    mag[::7] = 0
    grad = torch.from_numpy((mag * np.where(np.arange(n) % 2, 1, -1)).astype(F)).cuda()
    kge.AdamW([p], [st], weight_decay=0.0, seed=0xABCDEF0123456789, tag=9).step([grad], 1e-3, 1)
    m, v = _moments(np.zeros(n, F), np.zeros(n, F), grad.cpu().numpy())
    w = _philox(n, 0, 1, 0xABCDEF0123456789, 9)
    _check_codes(st.m, st.m_scales, m, "e4m3", (w & 0xFFFF) / 65536)
    _check_codes(st.v, st.v_scales, v, "e5m2", (w >> 16) / 65536)
    codes = st.v.cpu().numpy()
    assert (codes[v > 0] > 0).all() and (codes[v == 0] == 0).all() and bool((p[::7] == 1).all())


def test_stochastic_rounding_is_unbiased():
    """Moments that a step changes by far less than a spacing move on average as they should: after 400 steps on gradients of one size the means lie within six standard
    deviations of the exact moments, with the variance of a rounding at most spacing x change a step, spacing <= value / 4 (v) and value / 8 (m)."""
    n, steps = 1 << 16, 400
    p, st = torch.zeros(n, device="cuda"), kge.AdamWState.zeros(n, 8)
    opt = kge.AdamW([p], [st], weight_decay=0.0, seed=77)
    v = 0.0
    for s in range(1, steps + 1):
        opt.step([torch.full((n,), 1.0 if s <= 200 else 0.1, device="cuda")], 1e-3, s)
        g = 1.0 if s <= 200 else 0.1
        v = float(CFG["b2"]) * v + (1 - float(CFG["b2"])) * g * g
    got = _decode(st.v, st.v_scales, n, "e5m2")
    # v grows for 200 steps by 1e-3 each: variance below sum of v / 4 x 1e-3 <= 200 x 0.2 / 4 x 1e-3; then decays, adding as much again at most
    std = math.sqrt(2 * 200 * 0.2 / 4 * 1e-3)
    assert abs(got.mean() - v) < 6 * std / math.sqrt(n) + 400 * 2.0 ** -16 * v / 4
    assert got.std() < std


def test_the_update_in_a_graph_with_a_device_counter():
    sizes, bits = [3000, 64, 700], [8, 32, 8]
    a, _ = _run(sizes, bits, F32, True, key=90, step=1)
    b, _ = _run(sizes, bits, F32, True, key=90, step=1)
    mk = lambda ts: kge.AdamW([t[0] for t in ts], [t[2] for t in ts], shadows=[t[3] for t in ts], seed=4)       # noqa: E731
    one, two = mk(a), mk(b)
    grads = [t[1] for t in b]
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.step(grads, 1e-3, 2, step_counter=counter)
        kge.step_counter_add(counter)
    for i in range(4):
        for t in grads:
            t.copy_(torch.from_numpy(_rng(91, i, t.numel()).normal(size=t.numel()).astype(F)))
        one.step(grads, 1e-3, 2 + i)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            for s, t in ((x[0], y[0]), (x[3], y[3]), (x[2].m, y[2].m), (x[2].v, y[2].v)):
                assert torch.equal(s, t), i


@pytest.mark.parametrize("bits", [32, 8])
def test_beyond_32_bits(bits):
    n = (1 << 31) + 700
    p, grad = torch.ones(n, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    grad[-300:] = 0.5
    st = kge.AdamWState.zeros(n, bits)
    kge.AdamW([p], [st], weight_decay=0.0).step([grad], float(CFG["lr"]), 1)
    want = 1 - float(CFG["lr"]) / (1 + float(CFG["eps"]) / 0.5)
    assert bool((p[:-300][-5000:] == 1).all()) and bool((p[:5000] == 1).all())
    assert bool(((p[-300:].double() - want).abs() <= 4 * U).all())
    assert not bool(st.m[:1000].any()) and bool((st.m[n - 300:n] != 0).all()) and bool((st.v[n - 300:n] != 0).all())


def test_the_binding_refuses():
    p = torch.zeros(10, device="cuda")
    ok = kge.AdamW([p])
    for bad in [lambda: kge.AdamW([p.double()]), lambda: kge.AdamW([p.cpu()]), lambda: kge.AdamW([torch.zeros((4, 4), device="cuda").t()[:3]]), lambda: kge.AdamW([p], bits=16),
                lambda: kge.AdamW([p], [kge.AdamWState.zeros(11)]), lambda: kge.AdamW([p], shadows=[p]), lambda: kge.AdamW([p], weight_decay=[0.1, 0.1]),
                lambda: kge.AdamW([p], seed=-1), lambda: kge.AdamWState(p, p, p), lambda: ok.step([], 1e-3, 1), lambda: ok.step([p[:9]], 1e-3, 1),
                lambda: ok.step([p.cpu()], 1e-3, 1), lambda: ok.step([p.half()], 1e-3, 1), lambda: ok.step([p], 1e-3, 0), lambda: ok.step([p], 1e-3, 1, beta1=1.0),
                lambda: ok.step([p], 1e-3, 1, grad_scale=torch.ones(2, device="cuda")), lambda: kge.AdamW([p], weight_decay=-1.0).step([p], 1e-3, 1)]:
        with pytest.raises(kge.KgeError):
            bad()
    kge.AdamW([]).step([], 1e-3, 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_replaced_storage_is_found(bits):
    """A parameter whose storage has been replaced (p.data = ...) is updated where it is now, and its old storage left alone."""
    first = torch.linspace(-1, 1, 300, device="cuda")
    grad = torch.linspace(1, 2, 300, device="cuda")
    got, want = first.clone(), first.clone()
    shadow = [torch.zeros(300, dtype=BF16, device="cuda") for _ in range(2)]
    moved, still = kge.AdamW([got], bits=bits, shadows=shadow[:1]), kge.AdamW([want], bits=bits, shadows=shadow[1:])
    for step in (1, 2, 3):
        old = got.data
        kept = old.clone()
        got.data, shadow[0].data = old.clone(), torch.zeros_like(shadow[0])
        moved.step([grad], 1e-2, step)
        still.step([grad], 1e-2, step)
        assert torch.equal(got, want) and torch.equal(old, kept) and torch.equal(*shadow) and not torch.equal(got, kept)


def test_shared_tensors_are_refused():
    p = torch.zeros(1000, device="cuda")
    st = kge.AdamWState.zeros(1000)
    for bad in [lambda: kge.AdamW([p, p]), lambda: kge.AdamW([p[:600], p[500:]]), lambda: kge.AdamW([p, p.clone()], [st, st]), lambda: kge.AdamW([p], [kge.AdamWState(st.m, st.m)]),
                lambda: kge.AdamW([p], [kge.AdamWState(p, st.v)]), lambda: kge.AdamW([p], shadows=[p[:500].view(BF16)])]:
        with pytest.raises(kge.KgeError, match="overlap"):
            bad()
    kge.AdamW([p[:500], p[500:], torch.zeros(0, device="cuda"), torch.zeros(0, device="cuda")]).step([p[:500] + 1, p[500:] + 1, p[:0], p[:0]], 1e-3, 1)
    assert bool((p < 0).all())


def test_moments_on_the_grid_keep_their_codes():
    """Moments that a step halves exactly: the scale of a block falls by one and no code changes, whatever the random number - of four million for each moment every value of
    sixteen bits, 0 among them, comes up about 64 times - and whatever the block's scale."""
    blocks = 1 << 15
    n, g = 128 * blocks, _rng(95)
    codes = {}
    for k, top in (("m", 0x7e), ("v", 0x7b)):
        c = g.integers(0, top + 1, size=(blocks, 128)).astype(np.uint8)
        c[:, 0] = top                                             # (1.75 times the largest power of two: the block's scale follows from it)
        if k == "m":
            c[:, 1:] |= (g.integers(0, 2, size=(blocks, 127)) << 7).astype(np.uint8)
            c[c == 0x80] = 0                                      # (no zeros with a sign)
        codes[k] = torch.from_numpy(c.reshape(-1)).cuda()
    ms, vs = (torch.from_numpy((2 + np.arange(blocks) * 7919 % span).astype(np.uint8)).cuda() for span in (245, 238))
    st = kge.AdamWState(codes["m"].clone(), codes["v"].clone(), ms.clone(), vs.clone())
    p = torch.zeros(n, device="cuda")
    kge.AdamW([p], [st], weight_decay=0.0, seed=5).step([torch.zeros(n, device="cuda")], 0.0, 1, beta1=0.5, beta2=0.5)
    assert torch.equal(st.m_scales, ms - 1) and torch.equal(st.v_scales, vs - 1)
    assert torch.equal(st.m, codes["m"]), int((st.m != codes["m"]).sum())
    assert torch.equal(st.v, codes["v"]), int((st.v != codes["v"]).sum())


def _words(n, tensor, step, seed, tag):
    """_philox on whole arrays."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.arange(-(-n // 4), dtype=np.uint64)] + [np.full(-(-n // 4), w, dtype=np.uint64) for w in (tensor, step, tag)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [p1 >> half ^ c[1] ^ np.uint64(k[0]), p1 & low, p0 >> half ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=1).reshape(-1)[:n]


FORMATS = {"e4m3": (3, -6, 8, 0x7e), "e5m2": (2, -14, 15, 0x7b)}        # mantissa bits, exponents of the smallest and largest normal numbers, largest code


@pytest.mark.parametrize("gdt", [F32, BF16])
@pytest.mark.parametrize("n", [1000, 70_001])
def test_codes_by_the_generator(n, gdt):
    """With q the value in units of the spacing at its place, in 64 bits, and u its random number: floor(q + u), or one less where q + u is less than 2^-19 above that (the quotient by
    the scale is up to so much low), but never less than floor(q)."""
    assert np.array_equal(_words(101, 2, 3, 0xABCDEF0123456789, 9), _philox(101, 2, 3, 0xABCDEF0123456789, 9))
    ts, _ = _run([n, n], [8, 8], gdt, False, key=96)
    for i, (_, grad, st, _, m, v) in enumerate(ts):
        m, v = _moments(m, v, grad.float().cpu().numpy())
        w = _words(n, i, 3, 0xABCDEF0123456789, 9)
        for codes, scales, x, fmt, u in ((st.m, st.m_scales, m, "e4m3", w & np.uint64(0xFFFF)), (st.v, st.v_scales, v, "e5m2", w >> np.uint64(16))):
            bits, emin, _, top = FORMATS[fmt]
            s = scales.cpu().numpy().astype(np.int64)
            assert s[:-(-n // 128)].tolist() == [_byte(x[at:at + 128], fmt) for at in range(0, n, 128)]
            t = np.abs(x.astype(np.float64)) * 2.0 ** (127.0 - s[np.arange(n) // 128])
            e = np.maximum(np.frexp(t)[1] - 1, emin)
            q = t * 2.0 ** (bits - e)
            sums = q + u.astype(np.float64) / 65536
            least = np.where((x > 0) & (fmt == "e5m2"), 1, 0)
            code = lambda k: np.maximum(np.minimum(((e - emin) << bits) + k.astype(np.int64), top), least)      # noqa: E731
            high, low = code(np.floor(sums)), code(np.maximum(np.floor(sums - 2.0 ** -19), np.floor(q)))
            got = codes.cpu().numpy()[:n].astype(np.int64)
            assert np.array_equal(got >> 7, np.signbit(x))
            assert ((got & 0x7f == high) | (got & 0x7f == low)).all() and (high != low).mean() < 1e-4


def _elementary(x, fmt, rnd):
    """(codes, scale bytes) of fp32 values by elementary operations of torch on the GPU: powers of two, products, a sum and floor."""
    bits, emin, emax, top = FORMATS[fmt]
    x = x.view(-1, 128)
    mag = x.abs()
    mant, expo = torch.frexp(mag.amax(dim=1))
    s = (expo - 1 - emax + (mant > 0.875).int() + 127).clamp(min=0)
    a = (127 - s) // 2
    t = torch.ldexp(torch.ldexp(mag, a.unsqueeze(1)), (127 - s - a).unsqueeze(1))
    e = (torch.frexp(t)[1] - 1).clamp(min=emin)
    k = torch.floor(torch.ldexp(t, bits - e) + (rnd / 65536).view(-1, 128))
    code = (((e - emin) << bits) + k.int()).clamp(max=top)
    if fmt == "e5m2":
        code = torch.where((mag > 0) & (code == 0), 1, code)
    return (code | torch.signbit(x).int() << 7).view(-1).to(torch.uint8), s.to(torch.uint8)


def test_codes_of_elementary_steps():
    """Four million moments of each kind, in blocks of magnitudes 2^-90 to 2^40: a few of them lie on the border exactly."""
    blocks = 1 << 15
    n, g = 128 * blocks, _rng(97)
    grad = torch.from_numpy((g.normal(size=(blocks, 128)) * 2.0 ** g.uniform(-45, 20, size=(blocks, 1))).astype(F).reshape(-1)).cuda()
    p, st = torch.zeros(n, device="cuda"), kge.AdamWState.zeros(n, 8)
    kge.AdamW([p], [st], weight_decay=0.0, seed=0xABCDEF0123456789, tag=9).step([grad], 1e-3, 3)
    w = torch.from_numpy(_words(n, 0, 3, 0xABCDEF0123456789, 9).astype(np.int64)).cuda()
    for codes, scales, x, fmt, rnd in ((st.m, st.m_scales, grad * float(F(1) - CFG["b1"]), "e4m3", w & 0xFFFF), (st.v, st.v_scales, grad * grad * float(F(1) - CFG["b2"]), "e5m2", w >> 16)):
        want, s = _elementary(x, fmt, rnd.float())
        assert torch.equal(scales, s)
        off = (codes != want) & (rnd != 0)                        # (beside a random number of 0 the scale is divided out exactly)
        assert not bool(off.any()), (fmt, int(off.sum()))
