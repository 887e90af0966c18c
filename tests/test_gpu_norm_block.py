"""Norms around a block with gate and residual scale, forward and backward, against plain implementations in 64 bits on the CPU.

Tolerances follow each result's roundings: eps / 2 of the output's type, 2^-24 for every fp32 operation, and for a sum of n terms (n_add + 2) 2^-24 of the sum
of their magnitudes, n_add the longest chain of additions that a term goes through."""
import numpy as np
import pytest
import torch

import paper_2211_12281_amd as kge

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
CHAIN = 48                                  # of a row's sum: sixteen elements of a thread, six steps of a wave, sixteen waves, and the operations around
EPS = 1e-5


def _rng(*key):
    return np.random.default_rng([int(k) for k in key])


def _values(shape, dtype, *key, std=1.0, mean=0.0):
    return (torch.from_numpy(_rng(*key).normal(size=shape)) * std + mean).to(dtype)


def _padded(t, pad):
    """The same values on the GPU in rows that are `pad` elements longer, so that they start anywhere."""
    if t is None or pad == 0:
        return None if t is None else t.cuda()
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, pad // 2:pad // 2 + t.shape[1]] = t.cuda()
    return wide[:, pad // 2:pad // 2 + t.shape[1]]


def _within(got, want, tol, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]} +- {tol[bad][0]}"


class Case:
    """Inputs of one block."""

    def __init__(self, rows, dim, kind, s, b, post=True, pre=True, scale=True, gate_rows=0, y=True, bias=True, weight=True, key=0, mean=0.0):
        self.rows, self.dim, self.kind, self.s, self.b, self.gate_rows = rows, dim, kind, s, b, gate_rows
        v = lambda i, std, m: _values(dim, F32, key, i, dim, std=std, mean=m)            # noqa: E731
        self.x = _values((rows, dim), s, key, 1, rows, dim, mean=mean)
        self.y = _values((rows, dim), b, key, 2, rows, dim, std=3.0, mean=mean) if y else None
        mk = lambda i, on: [v(i, 0.3, 1.0) if weight else None, v(i + 1, 0.3, 0.0) if bias else None] if on else None     # noqa: E731
        self.post, self.pre = mk(10, post and y), mk(20, pre)
        self.scale = v(30, 0.2, 0.5) if scale and y else None
        self.groups = -(-rows // gate_rows) if gate_rows and y else 0
        self.gate = _values((self.groups, dim), b, key, 3, rows, dim) if gate_rows and y else None
        self.dh, self.dz = _values((rows, dim), s, key, 4, rows, dim), _values((rows, dim), b, key, 5, rows, dim) if pre else None

    def args(self, pad=0):
        n = lambda p: None if p is None else kge.Norm(self.kind, *(None if t is None else t.cuda() for t in p), eps=EPS)    # noqa: E731
        return dict(post=n(self.post), pre=n(self.pre), scale=None if self.scale is None else self.scale.cuda(), gate=_padded(self.gate, pad),
                    gate_rows=self.gate_rows or None)

    def per_row(self, t):
        return t[torch.arange(self.rows) // self.gate_rows]


def _hat(x, ex, kind):
    """(x^, its error, r, r's relative error) of rows that are known to ex"""
    d = x.shape[1]
    mean = lambda t: t.mean(dim=1, keepdim=True)                                             # noqa: E731
    xc, e = x, ex
    if kind == "layer":
        xc = x - mean(x)
        e = ex + mean(ex) + (CHAIN + 2) * U * (x.abs() + mean(x.abs()))
    var = mean(xc ** 2)
    evar = (CHAIN + 4) * U * var + mean(2 * xc.abs() * e + e ** 2)
    r = (var + float(np.float32(EPS))) ** -0.5
    rel = 0.5 * evar / (var + EPS) + 4 * U
    assert d == xc.shape[1]
    hat = xc * r
    return hat, e * r + hat.abs() * (rel + 2 * U), r, rel


def _affine(hat, e, p):
    w = 1.0 if p[0] is None else p[0].double()
    b = 0.0 if p[1] is None else p[1].double()
    out = hat * w + b
    return out, e * abs(w) + 2 * U * ((hat * w).abs() + abs(b))


def _forward(c):
    """{name: (value, tolerance)}"""
    h, eh, out = c.x.double(), torch.zeros(c.rows, c.dim, dtype=torch.float64), {}
    if c.y is not None:
        u, e = c.y.double(), torch.zeros_like(h)
        if c.post:
            u, e = _affine(*_hat(u, e, c.kind)[:2], c.post)
        f = torch.ones_like(u)
        if c.scale is not None:
            f = f * c.scale.double()
        if c.gate is not None:
            f = f * c.per_row(c.gate.double())
        eh = e * f.abs() + 3 * U * (u * f).abs()
        h = h + u * f
        eh = eh + U * h.abs()
        out["h"] = h, eh + HALF[c.s] * h.abs()
    if c.pre:
        z, e = _affine(*_hat(h, eh, c.kind)[:2], c.pre)
        out["z"] = z, e * (1 + HALF[c.b]) + HALF[c.b] * z.abs()
    return out


def _norm_bwd(t, et, hat, ehat, r, rel, kind):
    """Gradient of the rows from that of the normalised ones, t, known to et"""
    mean = lambda v: v.mean(dim=1, keepdim=True)                                             # noqa: E731
    c2, e2 = mean(t * hat), mean(et * hat.abs() + t.abs() * ehat) + (CHAIN + 2) * U * mean((t * hat).abs())
    c1, e1 = (mean(t), mean(et) + (CHAIN + 2) * U * mean(t.abs())) if kind == "layer" else (torch.zeros_like(c2), torch.zeros_like(c2))
    v = (t - c1 - hat * c2) * r
    e = (et + e1 + hat.abs() * e2 + ehat * c2.abs() + 4 * U * (t.abs() + c1.abs() + (hat * c2).abs())) * r
    return v, e * (1 + rel) + v.abs() * (rel + 2 * U)


def _backward(c):
    zero = torch.zeros(c.rows, c.dim, dtype=torch.float64)
    n = c.rows + 40                                                                          # additions of a column's sum
    out = {}

    def column(v, e):
        return v.sum(dim=0), e.sum(dim=0) + (n + 2) * U * v.abs().sum(dim=0)
    d, ed = c.dh.double(), zero
    if c.pre:
        hat, e, r, rel = _hat(c.x.double(), zero, c.kind)
        dz, w = c.dz.double(), 1.0 if c.pre[0] is None else c.pre[0].double()
        if c.pre[0] is not None:
            out["pre_weight"] = column(dz * hat, dz.abs() * e)
        if c.pre[1] is not None:
            out["pre_bias"] = column(dz, zero)
        v, ev = _norm_bwd(dz * w, U * (dz * w).abs(), hat, e, r, rel, c.kind)
        ed = ev + U * (d.abs() + v.abs())
        d = d + v
    out["x"] = d, ed * (1 + HALF[c.s]) + HALF[c.s] * d.abs()
    if c.y is None:
        return out
    hat, e, r, rel = (c.y.double(), zero, torch.ones_like(zero[:, :1]), torch.zeros_like(zero[:, :1])) if not c.post else _hat(c.y.double(), zero, c.kind)
    w = 1.0 if not c.post or c.post[0] is None else c.post[0].double()
    b = 0.0 if not c.post or c.post[1] is None else c.post[1].double()
    s = 1.0 if c.scale is None else c.scale.double()
    g = torch.ones_like(zero) if c.gate is None else c.per_row(c.gate.double())
    # the sums come as w A + b B, of magnitudes |w| sum |.| + |b| sum |.|
    term, eterm = d * (hat * w + b), (ed * hat.abs() + d.abs() * e + 2 * U * (d * hat).abs()) * abs(w) + (ed + U * d.abs()) * abs(b)
    mag = (d * hat).abs() * abs(w) + d.abs() * abs(b)

    def summed(v, ev, m, f):
        return f * v, abs(f) * (ev + (n + 6) * U * m)
    if c.gate is not None:
        where = torch.arange(c.rows) // c.gate_rows
        fold = lambda t: torch.zeros(c.groups, c.dim, dtype=torch.float64).index_add_(0, where, t)      # noqa: E731
        v, ev = summed(fold(term), fold(eterm), fold(mag), s)
        out["gate"] = v, ev * (1 + HALF[c.b]) + HALF[c.b] * v.abs()
    G = lambda t: (t * g).sum(dim=0)                                                          # noqa: E731
    A = lambda t: (t * g.abs()).sum(dim=0)                                                    # noqa: E731
    if c.scale is not None:
        out["scale"] = summed(G(term), A(eterm), A(mag), 1.0)
    if c.post and c.post[0] is not None:
        out["post_weight"] = summed(G(d * hat), A(ed * hat.abs() + d.abs() * e + 2 * U * (d * hat).abs()), A((d * hat).abs()), s)
    if c.post and c.post[1] is not None:
        out["post_bias"] = summed(G(d), A(ed + U * d.abs()), A(d.abs()), s)
    f = s * g * w
    t, et = d * f, ed * abs(f) + 4 * U * (d * f).abs()
    v, ev = _norm_bwd(t, et, hat, e, r, rel, c.kind) if c.post else (t, et)
    out["y"] = v, ev * (1 + HALF[c.b]) + HALF[c.b] * v.abs()
    return out


def _check_forward(c, pad=0):
    want = _forward(c)
    out = {}
    if c.y is not None:
        out["out_h"] = _padded(torch.zeros((c.rows, c.dim), dtype=c.s), pad)
    if c.pre:
        out["out_z"] = _padded(torch.zeros((c.rows, c.dim), dtype=c.b), pad)
    h, z = kge.norm_block(_padded(c.x, pad), _padded(c.y, pad), dtype=c.b if c.y is None else None, **out, **c.args(pad))
    for k, t in (("h", h), ("z", z)):
        if k in want:
            _within(t, *want[k], k)
    for t in out.values():
        if pad:                                                   # what lies between the rows stays
            assert bool(torch.isnan(t._base[:, :pad // 2]).all()) and bool(torch.isnan(t._base[:, pad // 2 + c.dim:]).all())


def _check_backward(c, pad=0):
    want = _backward(c)
    got = kge.norm_block_bwd(_padded(c.x, pad), _padded(c.y, pad), dh=_padded(c.dh, pad), dz=_padded(c.dz, pad), **c.args(pad))
    assert set(got) == set(want)
    for k, (v, tol) in want.items():
        _within(got[k], v, tol, k)


TYPES = [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)]
SHAPES = [(1, 1, 0), (3, 7, 1), (5, 64, 0), (70, 129, 3), (33, 512, 0), (41, 513, 1), (130, 768, 0), (9, 1000, 2), (19, 2049, 1), (6, 4097, 0), (3, 8191, 1),
          (2, 8192, 0), (40, 6000, 0), (50, 3500, 0), (1, 768, 0), (4500, 24, 0)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("s,b", TYPES)
@pytest.mark.parametrize("rows,dim,pad", SHAPES)
def test_norm_block(rows, dim, pad, s, b, kind):
    _check_forward(Case(rows, dim, kind, s, b, gate_rows=[0, 1, 3, rows][(rows + dim) % 4]), pad)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("s,b", TYPES)
@pytest.mark.parametrize("rows,dim,pad", SHAPES)
def test_norm_block_bwd(rows, dim, pad, s, b, kind):
    _check_backward(Case(rows, dim, kind, s, b, gate_rows=[0, 1, 3, rows][(rows + dim) % 4], key=1), pad)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,dim", [(1, 40), (37, 72), (37, 700), (300, 1100), (20_011, 16)])
@pytest.mark.parametrize("gate_rows", [1, 2, 5, 16, 17, 37, 100, 1 << 40])
def test_gates_of_groups(rows, dim, kind, gate_rows):
    c = Case(rows, dim, kind, F32, F32, gate_rows=gate_rows, key=2)
    _check_forward(c)
    _check_backward(c)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("s,b", TYPES)
@pytest.mark.parametrize("rows,dim", [(9_000, 128), (2_000, 65), (8_501, 250), (900, 256), (3_000, 257), (35_000, 60)])
@pytest.mark.parametrize("gate_rows", [0, 1, 2, 150])
def test_narrow_rows_share_a_wave(rows, dim, gate_rows, s, b, kind):
    c = Case(rows, dim, kind, s, b, gate_rows=gate_rows, key=4)
    _check_forward(c, 1)
    _check_backward(c, 1)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("s,b", TYPES)
@pytest.mark.parametrize("rows,dim", [(5, 1025), (300, 1537), (31, 2000), (77, 2048), (12, 2560), (9000, 2561), (64, 2900), (7, 3333)])
def test_rows_of_two_waves(rows, dim, s, b, kind):
    _check_forward(Case(rows, dim, kind, s, b, gate_rows=[0, 1, 3, rows][rows % 4], key=5), 1)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("s,b", TYPES)
@pytest.mark.parametrize("rows,dim", [(513, 3400), (1111, 4096), (701, 8001), (515, 5000), (512, 4000)])
def test_pairs_of_wide_rows(rows, dim, s, b, kind):
    _check_forward(Case(rows, dim, kind, s, b, gate_rows=[0, 1, 3, rows][rows % 4], key=6), 1)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("parts", [dict(y=False), dict(pre=False), dict(post=False), dict(post=False, pre=False), dict(scale=False), dict(post=False, scale=False),
                                   dict(bias=False), dict(weight=False), dict(weight=False, bias=False, scale=False)])
@pytest.mark.parametrize("gate_rows", [0, 1, 9])
def test_parts_may_be_absent(kind, parts, gate_rows):
    c = Case(53, 136, kind, F32, BF16, gate_rows=0 if parts.get("y") is False else gate_rows, key=3, **parts)
    if c.y is not None and not c.post and c.scale is None and c.gate is None and not c.pre:
        pytest.skip("nothing to do")
    _check_forward(c)
    _check_backward(c)


def test_a_mean_far_from_zero():
    """Deviations are taken from the mean before they are squared."""
    c = Case(20, 768, "layer", F32, F32, key=4, mean=1000.0)
    _check_forward(c)
    _check_backward(c)


def test_without_a_stream_without_h_and_without_dh():
    c = Case(12, 300, "rms", F32, F32, gate_rows=4, key=5)
    c.x = torch.zeros_like(c.x)
    want = _forward(c)
    h, z = kge.norm_block(None, c.y.cuda(), **c.args())
    _within(h, *want["h"])
    none, z2 = kge.norm_block(None, c.y.cuda(), want_h=False, **c.args())
    assert none is None and torch.equal(z, z2)
    c.x, c.dh = _values(c.x.shape, F32, 55), torch.zeros_like(c.dh)
    want = _backward(c)
    got = kge.norm_block_bwd(c.x.cuda(), c.y.cuda(), dz=c.dz.cuda(), **c.args())
    for k, (v, tol) in want.items():
        _within(got[k], v, tol, k)


def test_in_place():
    c = Case(400, 96, "layer", F32, BF16, gate_rows=7, key=6)
    x = c.x.cuda()
    h, z = kge.norm_block(c.x.cuda(), c.y.cuda(), **c.args())
    h2, z2 = kge.norm_block(x, c.y.cuda(), out_h=x, **c.args())
    assert h2 is x and torch.equal(h, h2) and torch.equal(z, z2)
    got = kge.norm_block_bwd(h, c.y.cuda(), dh=c.dh.cuda(), dz=c.dz.cuda(), **c.args())
    dh = c.dh.cuda()
    got2 = kge.norm_block_bwd(h, c.y.cuda(), dh=dh, dz=c.dz.cuda(), out={"x": dh}, **c.args())
    assert got2["x"] is dh
    for k in got:
        assert torch.equal(got[k], got2[k]), k


@pytest.mark.parametrize("gate_rows", [0, 1, 3, 90])
def test_wanted_gradients_are_the_same_alone_and_accumulated(gate_rows):
    c = Case(180, 200, "layer", F32, F32, gate_rows=gate_rows, key=7)
    call = lambda **k: kge.norm_block_bwd(c.x.cuda(), c.y.cuda(), dh=c.dh.cuda(), dz=c.dz.cuda(), **c.args(), **k)     # noqa: E731
    whole = call()
    for k in whole:
        (alone,) = call(want=[k]).values()
        assert torch.equal(alone, whole[k]), k
    sums = ["scale", "post_weight", "post_bias", "pre_weight", "pre_bias"]
    old = {k: _values(200, F32, 77, i).cuda() for i, k in enumerate(sums)}
    got = call(want=sums, out={k: t.clone() for k, t in old.items()}, accumulate=True)
    for k in sums:
        want = old[k].double().cpu() + whole[k].double().cpu()
        _within(got[k], want, 2 * U * (want.abs() + whole[k].double().cpu().abs()), k)
    ws = kge.Workspace()
    ws.get(1 << 22)
    for k, t in call(ws=ws).items():
        assert torch.equal(t, whole[k]), k


def test_no_rows():
    p = kge.Norm("layer", torch.ones(64, device="cuda"), torch.zeros(64, device="cuda"))
    x = torch.empty((0, 64), device="cuda")
    h, z = kge.norm_block(x, x, post=p, pre=p, gate=x, gate_rows=3)
    assert h.shape == z.shape == (0, 64)
    got = kge.norm_block_bwd(x, x, dh=x, dz=x, post=p, pre=p, gate=x, gate_rows=3)
    assert got["x"].shape == (0, 64) and got["gate"].shape == (0, 64) and not bool(got["pre_weight"].any()) and not bool(got["post_bias"].any())
    old = torch.ones(64, device="cuda")
    got = kge.norm_block_bwd(x, dz=x, pre=p, want=["pre_weight"], out={"pre_weight": old}, accumulate=True)
    assert bool((old == 1).all())


def test_what_is_not_finite_stays_in_its_row():
    c = Case(9, 520, "layer", F32, F32, gate_rows=1, key=8)
    c.x[2, 5], c.y[4, 519], c.y[6, 0] = float("inf"), float("nan"), float("-inf")
    h, z = (t.cpu() for t in kge.norm_block(c.x.cuda(), c.y.cuda(), **c.args()))
    bad = torch.isnan(z).any(dim=1)
    assert bad.tolist() == [i in (2, 4, 6) for i in range(9)] and bool(torch.isnan(z[bad]).all())
    got = kge.norm_block_bwd(c.x.cuda(), c.y.cuda(), dh=c.dh.cuda(), dz=c.dz.cuda(), want=["x", "y"], **c.args())
    assert torch.isnan(got["x"]).any(dim=1).tolist() == [i == 2 for i in range(9)]
    assert torch.isnan(got["y"]).any(dim=1).tolist() == [i in (2, 4, 6) for i in range(9)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate_rows", [0, 1, 4])
def test_gradients_against_differences(kind, gate_rows):
    """Central differences of the 64-bit forward pass along a random direction of every input."""
    c = Case(10, 48, kind, F32, F32, gate_rows=gate_rows, key=9)
    fwd = _forward(c)
    cz, ch = _values((10, 48), F32, 91), _values((10, 48), F32, 92)
    h32 = fwd["h"][0].float()
    got = kge.norm_block_bwd(h32.cuda(), c.y.cuda(), dh=ch.cuda(), dz=cz.cuda(), **c.args())
    leaves = {"x": "x", "y": "y", "scale": "scale", "post_weight": ("post", 0), "post_bias": ("post", 1), "pre_weight": ("pre", 0), "pre_bias": ("pre", 1)}
    if gate_rows:
        leaves["gate"] = "gate"

    def loss():
        f = _forward(c)
        return float((f["h"][0] * ch.double()).sum() + (f["z"][0] * cz.double()).sum())
    for i, (name, at) in enumerate(leaves.items()):
        old = getattr(c, at) if isinstance(at, str) else getattr(c, at[0])[at[1]]
        v = _values(old.shape, torch.float64, 93, i)
        put = lambda t: setattr(c, at, t) if isinstance(at, str) else getattr(c, at[0]).__setitem__(at[1], t)       # noqa: E731
        step = 1e-4
        put(old.double() + step * v)
        up = loss()
        put(old.double() - step * v)
        down = loss()
        put(old)
        g = got[name].double().cpu()
        slope = (up - down) / (2 * step)
        # third derivatives times step^2 (1e-8), h rounded to fp32, and fp32 gradients
        assert abs(float((g * v).sum()) - slope) <= 1e-5 * float((g * v).abs().sum()) + 1e-6, name


def test_a_captured_pass_is_replayed():
    c = Case(700, 256, "layer", F32, BF16, gate_rows=50, key=10)
    args, ws = c.args(), kge.Workspace()
    x, y, dh, dz = c.x.cuda(), c.y.cuda(), c.dh.cuda(), c.dz.cuda()

    def both(ws=None):
        h, z = kge.norm_block(x, y, **args)
        return [h, z, *kge.norm_block_bwd(h, y, dh=dh, dz=dz, ws=ws, **args).values()]
    with pytest.raises(kge.KgeError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            kge.norm_block_bwd(x, y, dh=dh, dz=dz, **args)
    torch.cuda.synchronize()
    ws.get(64 << 20)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(ws)
    for i in range(4):
        x.copy_(_values(c.x.shape, F32, 100, i))
        want = both()
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i


def test_beyond_32_bits():
    rows, dim = (1 << 21) + 40, 1024                             # rows of 4.3 GB
    x = torch.zeros((rows, dim), dtype=BF16, device="cuda")
    last = _values((3, dim), BF16, 11)
    x[-3:] = last.cuda()
    w = _values(dim, F32, 12, mean=1.0)
    _, z = kge.norm_block(x, pre=kge.Norm("rms", w.cuda(), eps=EPS))
    hat, e, _, _ = _hat(last.double(), torch.zeros(3, dim, dtype=torch.float64), "rms")
    want = hat * w.double()
    _within(z[-3:], want, e * w.double().abs() + want.abs() * (2.0 ** -8 + 2 * U))
    assert not bool(z[:1000].any())
    got = kge.norm_block_bwd(x, dz=z, pre=kge.Norm("rms", w.cuda(), eps=EPS), out={"x": x}, dh=x, want=["x", "pre_weight"])
    zz = z[-3:].double().cpu()
    _within(got["pre_weight"], (zz * hat).sum(0), (zz.abs() * e).sum(0) + 60 * U * (zz * hat).abs().sum(0))


def test_the_binding_refuses():
    x = torch.zeros((4, 8), device="cuda")
    n = kge.Norm("rms", torch.ones(8, device="cuda"))
    for bad in [dict(pre=kge.Norm("rms", torch.ones(9, device="cuda"))), dict(), dict(pre=n, scale=torch.ones(8, device="cuda")),
                dict(y=x, gate=x[:3], gate_rows=3), dict(y=x, gate=x[:2]), dict(y=x.bfloat16(), gate=x, gate_rows=1), dict(y=x, scale=torch.ones(7, device="cuda")),
                dict(y=x[:3], pre=n), dict(y=x, pre=kge.Norm("rms", eps=0.0)), dict(y=x, out_z=x), dict(pre=n, out_h=x), dict(y=x.cpu(), pre=n),
                dict(y=x, pre=n, dtype=BF16)]:
        with pytest.raises(kge.KgeError):
            kge.norm_block(x, **bad)
    for bad in [dict(dz=x), dict(pre=n), dict(dh=x, dz=x), dict(dz=x, pre=n, want=["gate"]), dict(dz=x, pre=n, accumulate=True),
                dict(dz=x, pre=n, out={"scale": x}), dict(dz=x, pre=n, want=["x"], out={"pre_weight": x[0]}), dict(dz=x[:2], pre=n)]:
        with pytest.raises(kge.KgeError):
            kge.norm_block_bwd(x, **bad)
    with pytest.raises(kge.KgeError):
        kge.Norm("batch")
    with pytest.raises(kge.KgeError):
        kge.norm_block(torch.zeros((1, 8193), device="cuda"), pre=kge.Norm())


def test_replaced_storage_is_found():
    """A norm's weight and bias are read where they are at the call (weight.data = ... replaces the storage)."""
    x, w, b = torch.randn(40, 96, device="cuda"), torch.randn(96, device="cuda"), torch.randn(96, device="cuda")
    n = kge.Norm("layer", w, b)
    kge.norm_block(x, pre=n)
    w.data, b.data = torch.randn(96, device="cuda"), torch.randn(96, device="cuda")
    fresh = kge.Norm("layer", w.clone(), b.clone())
    assert torch.equal(kge.norm_block(x, pre=n)[1], kge.norm_block(x, pre=fresh)[1])
    g, f = (kge.norm_block_bwd(x, dz=x, pre=k) for k in (n, fresh))
    assert all(torch.equal(g[k], f[k]) for k in ("x", "pre_weight", "pre_bias"))
    w.data = torch.randn(95, device="cuda")
    with pytest.raises(kge.KgeError):
        kge.norm_block(x, pre=n)


# Rows by which every workgroup of the backward pass is full, its teams take a second row, and gates of two rows give each team groups of its own; a shape for each number of
# waves and of groups of four columns that a lane of a row may have
FULL = [(4_201, 300), (3_101, 700), (2_101, 1000), (1_601, 1100), (1_101, 1800), (1_101, 2048), (801, 2500), (601, 3500), (301, 4501), (301, 8191), (301, 8192)]


def _backward_on_the_gpu(c):
    for k, t in vars(c).items():
        setattr(c, k, t.cuda() if torch.is_tensor(t) else [None if p is None else p.cuda() for p in t] if isinstance(t, list) else t)
    with torch.device("cuda"):
        want = _backward(c)
    got = kge.norm_block_bwd(c.x, c.y, dh=c.dh, dz=c.dz, **c.args())
    assert set(got) == set(want)
    for k, (v, tol) in want.items():
        _within(got[k], v.cpu(), tol.cpu(), k)


@pytest.mark.parametrize("s,b", TYPES)
@pytest.mark.parametrize("rows,dim", FULL)
@pytest.mark.parametrize("gate_rows", [0, 1, 2, 150])
def test_full_workgroups(rows, dim, gate_rows, s, b):
    _backward_on_the_gpu(Case(rows, dim, "layer" if (rows + gate_rows + (s is b)) % 2 else "rms", s, b, gate_rows=gate_rows, key=12))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,dim", FULL)
def test_full_workgroups_of_groups_with_an_odd_end(rows, dim, kind):
    """Groups of three rows, the last of which has one or two."""
    rows = rows * 8 // 5
    _backward_on_the_gpu(Case(rows + (rows % 3 == 0), dim, kind, F32, BF16, gate_rows=3, key=13))


@pytest.mark.parametrize("rows,dim,gate_rows", [(20, 72, 0), (20, 72, 20), (300, 100, 0), (300, 100, 1), (300, 100, 100), (2_000, 72, 2_000), (20_011, 16, 2), (3_101, 700, 2), (301, 8191, 2)])
def test_an_infinite_gradient_without_a_bias(rows, dim, gate_rows):
    """Sums that an infinity is in are infinite, whatever number of workgroups they come from: what a bias would be multiplied by does not count."""
    c = Case(rows, dim, "rms", F32, F32, pre=False, bias=False, gate_rows=gate_rows, key=14)
    r, k = 3, 5
    c.dh[r, k] = float("inf")
    got = kge.norm_block_bwd(None, c.y.cuda(), dh=c.dh.cuda(), want=["scale", "post_weight"] + (["gate"] if gate_rows else []), **c.args())
    g = float(c.gate[r // gate_rows, k]) if gate_rows else 1.0
    y, w, s = float(c.y[r, k]), float(c.post[0][k]), float(c.scale[k])
    at = {"scale": (k, g * w * y), "post_weight": (k, g * s * y)} | ({"gate": ((r // gate_rows, k), s * w * y)} if gate_rows else {})
    for name, (i, sign) in at.items():
        t = got[name].cpu()
        assert t[i] == np.copysign(np.inf, sign), (name, t[i])
        t[i] = 0
        assert bool(torch.isfinite(t).all()), name


@pytest.mark.parametrize("s,b", [(BF16, BF16), (F32, BF16)])
def test_rows_beyond_32_bits_in_all_tensors(s, b):
    """The last rows of tensors of 4.3 GB (fp32: 8.6), forward and backward, each tensor its own; the rows before them are zeros and add nothing to the sums."""
    c, rows, dim = Case(3, 1024, "layer", s, b, key=15), (1 << 21) + 40, 1024

    def behind_zeros(t):
        wide = torch.zeros((rows, dim), dtype=t.dtype, device="cuda")
        wide[-3:] = t.cuda()
        return wide
    x, y = behind_zeros(c.x), behind_zeros(c.y)
    h, z = kge.norm_block(x, y, **c.args())
    for k, t in (("h", h), ("z", z)):
        _within(t[-3:], *_forward(c)[k], k)
    del h, z
    dh = behind_zeros(c.dh)
    got = kge.norm_block_bwd(x, y, dh=dh, dz=behind_zeros(c.dz), out={"x": dh}, **c.args())
    for k, (v, tol) in _backward(c).items():
        _within(got[k][-3:] if k in ("x", "y") else got[k], v, tol, k)
    for k in ("x", "y"):
        for at in (0, (1 << 20) - 2, (1 << 21) - 2, rows - 10):
            assert not bool(got[k][at:at + 4].any()), (k, at)
