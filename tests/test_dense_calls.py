"""Refusals, workspace sizes and scratch space of the norms around a block, the 8-bit integer matrices and the dense AdamW: all of it is decided on the host,
before a GPU call (fake addresses: nothing dereferences them)."""
import ctypes as C

import pytest
import torch

import paper_2211_12281_amd.binding as b
from test_scratch_space import FakeStream, _at_once, on_the_host  # noqa: F401

OK = 0x10000000
INVALID, UNSUPPORTED, SMALL = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return b.load()


NORM = b.KgeNormT(0, 1e-5, OK, OK)


def _blk(**kw):
    a = dict(dim=64, stream_dtype=0, block_dtype=1, reserved=0, post=C.addressof(NORM), pre=C.addressof(NORM), scale=OK, gate=OK, gate_ld=64, gate_rows=2)
    a.update(kw)
    return b.KgeNormBlockT(*[a[f] for f, _ in b.KgeNormBlockT._fields_])


def _fwd(lib, blk=None, **kw):
    a = dict(x=OK, xld=64, y=OK, yld=64, rows=4, h=OK, hld=64, z=OK, zld=64)
    a.update(kw)
    s = _blk(**(blk or {}))
    return lib.kge_norm_block(C.byref(s), a["x"], a["xld"], a["y"], a["yld"], a["rows"], a["h"], a["hld"], a["z"], a["zld"], None)


def _bwd(lib, blk=None, grads=None, **kw):
    a = dict(h=OK, y=OK, dh=OK, dz=OK, ld=64, rows=4, dx=OK, dy=OK, ws=None, wsb=0)
    a.update(kw)
    s, g = _blk(**(blk or {})), b.KgeNormBlockGradsT(**{**dict(post_weight=OK, pre_bias=OK, gate=OK, gate_ld=64), **(grads or {})})
    ld = a["ld"]
    return lib.kge_norm_block_bwd(C.byref(s), a["h"], ld, a["y"], ld, a["dh"], ld, a["dz"], ld, a["rows"], a["dx"], ld, a["dy"], ld, C.byref(g), a["ws"], a["wsb"], None)


BAD_NORMS = [b.KgeNormT(2, 1e-5, OK, OK), b.KgeNormT(0, 0.0, OK, OK), b.KgeNormT(0, -1.0, OK, OK), b.KgeNormT(0, float("nan"), OK, OK), b.KgeNormT(0, float("inf"), OK, OK),
             b.KgeNormT(0, 1e-5, OK + 2, OK), b.KgeNormT(1, 1e-5, OK, OK + 1)]
BAD_BLK = [dict(dim=0), dict(dim=-4), dict(stream_dtype=2), dict(block_dtype=-1), dict(reserved=1), dict(scale=OK + 2), dict(gate=OK + 1), dict(gate_ld=63),
           dict(gate_rows=0), dict(gate_rows=-1), *[{k: C.addressof(n)} for k in ("post", "pre") for n in BAD_NORMS]]


@pytest.mark.parametrize("i", range(len(BAD_BLK)))
def test_norm_block_refuses_blocks(lib, i):
    assert _fwd(lib, BAD_BLK[i]) == INVALID and _bwd(lib, BAD_BLK[i]) == INVALID
    assert lib.kge_norm_block_bwd_workspace_bytes(C.byref(_blk(**BAD_BLK[i])), 4) == 0


@pytest.mark.parametrize("bad", [dict(y=None), dict(x=None, y=None), dict(z=None), dict(xld=63), dict(yld=63), dict(hld=63), dict(zld=63), dict(rows=-1), dict(rows=1 << 31),
                                 dict(x=OK + 2), dict(y=OK + 1), dict(h=OK + 2), dict(z=OK + 1), dict(xld=1 << 31), dict(blk=dict(pre=None)),
                                 dict(blk=dict(pre=None), z=None, h=None), dict(blk=dict(post=None, scale=None, gate=None), y=None)])
def test_norm_block_refuses(lib, bad):
    assert _fwd(lib, **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(y=None), dict(h=None), dict(dz=None), dict(ld=63), dict(rows=-1), dict(h=OK + 2), dict(dy=OK + 1), dict(blk=dict(pre=None)),
                                 dict(blk=dict(pre=None), dz=None, dh=None, grads=dict(pre_bias=None)), dict(grads=dict(scale=OK), blk=dict(scale=None)),
                                 dict(grads=dict(accumulate=2)), dict(grads=dict(reserved=1)), dict(grads=dict(post_bias=OK + 2)), dict(grads=dict(gate_ld=63)),
                                 dict(blk=dict(gate=None)), dict(blk=dict(post=None, scale=None, gate=None), y=None, grads=dict(post_weight=None, gate=None))])
def test_norm_block_bwd_refuses(lib, bad):
    assert _bwd(lib, **bad) == INVALID


def test_norm_block_limits(lib):
    wide = dict(dim=8193, gate_ld=8193)
    assert _fwd(lib, wide, xld=8193, yld=8193, hld=8193, zld=8193) == UNSUPPORTED
    assert _bwd(lib, wide, dict(gate_ld=8193), ld=8193) == UNSUPPORTED
    assert _fwd(lib, rows=0) == 0 and _bwd(lib, rows=0, grads=dict(post_weight=None, pre_bias=None)) == 0
    assert _fwd(lib, rows=0, x=None, y=None, h=None, z=None) == 0
    size = lib.kge_norm_block_bwd_workspace_bytes
    need = size(C.byref(_blk()), 100)
    assert need > 256 and _bwd(lib, rows=100) == SMALL and _bwd(lib, rows=100, ws=OK + 8, wsb=255) == SMALL
    assert size(C.byref(_blk()), -1) == 0 and size(C.byref(_blk()), 1 << 31) == 0
    for gate_rows in (1, 2, 3, 100, 1 << 40):
        for dim in (1, 64, 600, 1500, 4000, 8192):
            blk = _blk(dim=dim, gate_ld=dim, gate_rows=gate_rows)
            sizes = [size(C.byref(blk), r) for r in (*range(0, 200, 7), 4096, 4097, 24_576, 1 << 20, (1 << 31) - 1)]
            assert sizes == sorted(sizes) and sizes[-1] < 1 << 30


def _q(rows=256, cols=300, **kw):
    a = dict(rows=rows, cols=cols, codes=OK, ld=-(-cols // 128) * 128, scales=OK)
    a.update(kw)
    return b.KgeRowwiseT(*[a[f] for f, _ in b.KgeRowwiseT._fields_])


BAD_Q = [dict(codes=None), dict(scales=None), dict(ld=256), dict(ld=392), dict(codes=OK + 8), dict(scales=OK + 2), dict(rows=-1), dict(ld=1 << 32)]


@pytest.mark.parametrize("bad", BAD_Q)
def test_rowwise_refuses_layouts(lib, bad):
    assert lib.kge_quantize_rowwise(OK, 0, 256, 300, 300, C.byref(_q(**bad)), None, None, 0, None) == INVALID
    assert lib.kge_quantize_rowwise(OK, 0, 300, 256, 256, None, C.byref(_q(**bad)), OK, 1 << 20, None) == INVALID
    assert lib.kge_matmul_rowwise(C.byref(_q(**bad)), None, 256, C.byref(_q(512)), 0, OK, 0, 512, None, 0, None) == INVALID
    assert lib.kge_matmul_rowwise(C.byref(_q(512)), None, 512, C.byref(_q(**bad)), 0, OK, 0, 256, None, 0, None) == INVALID


def test_quantize_rowwise_refuses(lib):
    good, col = _q(), _q(300, 256)
    call = lambda x=OK, dt=0, rows=256, cols=300, ld=300, r=good, c=None, ws=None, wsb=0: lib.kge_quantize_rowwise(   # noqa: E731
        x, dt, rows, cols, ld, C.byref(r) if r else None, C.byref(c) if c else None, ws, wsb, None)
    for bad in [dict(x=None), dict(dt=2), dict(rows=255), dict(cols=299), dict(ld=299), dict(r=None), dict(x=OK + 2), dict(c=good), dict(rows=-1), dict(ld=1 << 31)]:
        assert call(**bad) == INVALID, bad
    need = lib.kge_quantize_rowwise_workspace_bytes(600, 300)
    tall = dict(rows=600, r=_q(600), c=_q(300, 600))
    assert need > 300 * 4 and call(**tall) == SMALL and call(**tall, ws=OK + 8, wsb=need - 256) == SMALL
    assert lib.kge_quantize_rowwise_workspace_bytes(512, 300) == 256 and col.rows == 300
    assert call(rows=131_072, cols=2, ld=2, r=None, c=_q(2, 131_072), ws=OK, wsb=1 << 30) == UNSUPPORTED
    assert call(cols=131_072, rows=2, ld=131_072, r=_q(2, 131_072)) == UNSUPPORTED
    assert call(rows=0, cols=300, r=_q(0), x=None) == 0
    size = lib.kge_quantize_rowwise_workspace_bytes
    assert size(-1, 1) == 0 and size(1, 1 << 31) == 0


def test_matmul_rowwise_refuses(lib):
    def mm(a=None, bb=None, **kw):
        v = dict(rows=None, m=256, acc=0, out=OK, dt=0, ld=512, ws=None, wsb=0)
        v.update(kw)
        return lib.kge_matmul_rowwise(C.byref(a or _q()), v["rows"], v["m"], C.byref(bb or _q(512)), v["acc"], v["out"], v["dt"], v["ld"], v["ws"], v["wsb"], None)
    for bad in [dict(m=255), dict(m=-1, rows=OK), dict(rows=OK + 2), dict(acc=2), dict(out=None), dict(dt=5), dict(ld=511), dict(out=OK + 2), dict(ld=1 << 31),
                dict(bb=_q(512, 301))]:
        assert mm(**bad) == INVALID, bad
    assert mm(bb=_q(0)) == 0 and mm(a=_q(0), m=0, out=None) == 0
    assert mm(a=_q(256, 131_072), bb=_q(512, 131_072)) == UNSUPPORTED
    assert mm(bb=_q((1 << 31) - 1, 300), a=_q(3), m=3, ld=(1 << 31) - 1) == UNSUPPORTED              # more workgroups than a grid holds
    size = lib.kge_matmul_rowwise_workspace_bytes
    assert size(-1, 1, 1) == 0 and size(1, 1 << 31, 1) == 0 and size(1, 2048, 2048) >= 256
    assert size(1024, 768, 24576) >= 2 * 4 * 1024 * 768


def _adamw(lib, cfg=None, count=1, **kw):
    a = dict(param_f32=OK, param_bf16=None, grad=OK, grad_dtype=0, state_bits=32, m=OK, v=OK, m_scales=None, v_scales=None, n=10, weight_decay=0.1, reserved=0)
    a.update(kw)
    t = b.KgeAdamwTensorT(*[a[f] for f, _ in b.KgeAdamwTensorT._fields_])
    c = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, step_counter=None)
    more = {k: v for k, v in (cfg or {}).items() if k not in c}
    c.update({k: v for k, v in (cfg or {}).items() if k in c})
    s = b.KgeAdamwCfgT(b.KgeAdamCfgT(*c.values()), **more)
    return lib.kge_adamw(C.byref(t), count, C.byref(s), None)


@pytest.mark.parametrize("bad", [dict(param_f32=None), dict(grad=None), dict(m=None), dict(v=None), dict(grad_dtype=2), dict(state_bits=16), dict(n=-1), dict(n=1 << 34),
                                 dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(reserved=1), dict(param_f32=OK + 2), dict(param_bf16=OK + 1), dict(grad=OK + 2),
                                 dict(grad=OK + 1, grad_dtype=1), dict(m=OK + 2), dict(state_bits=8), dict(state_bits=8, m_scales=OK, v_scales=OK, m=OK + 8),
                                 dict(state_bits=8, m_scales=OK), dict(cfg=dict(step=0)), dict(cfg=dict(beta1=1.0)), dict(cfg=dict(beta2=-0.1)), dict(cfg=dict(eps=-1.0)),
                                 dict(cfg=dict(lr=float("nan"))), dict(cfg=dict(reserved=1)), dict(cfg=dict(grad_scale=OK + 2)), dict(cfg=dict(step_counter=OK + 4)), dict(count=-2)])
def test_adamw_refuses(lib, bad):
    assert _adamw(lib, **bad) == INVALID
    assert lib.kge_adamw(None, 1, C.byref(b.KgeAdamwCfgT()), None) == INVALID


def test_adamw_of_nothing(lib):
    cfg = b.KgeAdamwCfgT(b.KgeAdamCfgT(1e-3, 0.9, 0.999, 1e-8, 1, None))
    assert lib.kge_adamw(None, 0, C.byref(cfg), None) == 0
    t = b.KgeAdamwTensorT(state_bits=32)
    assert lib.kge_adamw(C.byref(t), 1, C.byref(cfg), None) == 0


# Scratch space: of each call's own, of the stream that it runs on (the same stand-ins as for the other calls of the text side)
def _call_bwd(ws=None, stream=None):
    x = torch.zeros((5, 8))
    b.norm_block_bwd(x, dz=x, pre=b.Norm("rms", torch.ones(8)), ws=ws, stream=stream)


def _call_quantize(ws=None, stream=None):
    b.quantize_rowwise(torch.zeros((5, 8)), by="col", ws=ws, stream=stream)


def _call_matmul(ws=None, stream=None):
    q = b.Rowwise(torch.zeros((5, 128), dtype=torch.int8), torch.ones(5), 100)
    b.matmul_rowwise(q, q, ws=ws, stream=stream)


CALLS = [_call_bwd, _call_quantize, _call_matmul]


@pytest.fixture
def sizes(monkeypatch):
    monkeypatch.setattr(b, "_rowwise_bytes", lambda *a: 3 << 20)
    monkeypatch.setattr(b, "_matmul_rowwise_bytes", lambda *a: 3 << 20)


@pytest.mark.parametrize("one", CALLS)
@pytest.mark.parametrize("two", CALLS)
def test_calls_of_two_threads_hold_memory_of_their_own(monkeypatch, on_the_host, sizes, one, two):     # noqa: F811
    (p, n), (q, m) = _at_once(monkeypatch, [one, two])
    assert p + n <= q or q + m <= p


@pytest.mark.parametrize("call", CALLS)
def test_calls_take_memory_of_the_stream_they_run_on(monkeypatch, on_the_host, sizes, call):           # noqa: F811
    for stream in (None, FakeStream()):
        ((p, _),) = _at_once(monkeypatch, [lambda: call(stream=stream)])
        assert on_the_host[p] is stream


@pytest.mark.parametrize("call", CALLS)
def test_a_given_workspace_is_used(monkeypatch, on_the_host, sizes, call):                             # noqa: F811
    ws = b.Workspace()
    ((p, n),) = _at_once(monkeypatch, [lambda: call(ws=ws)])
    assert (p, n) == (ws.buf.data_ptr(), ws.buf.numel())


# Matrices without rows or columns
@pytest.mark.parametrize("rows", [0, 5, 600, 1 << 20])
def test_quantize_rowwise_of_no_columns(lib, rows):
    size = lib.kge_quantize_rowwise_workspace_bytes
    assert size(rows, 0) == size(0, rows) == 256
    by_col = _q(0, min(rows, 131_071), codes=None, scales=None)
    assert lib.kge_quantize_rowwise(None, 0, by_col.cols, 0, 0, None, C.byref(by_col), None, 0, None) == 0


def test_quantize_rowwise_of_nothing_both_ways(lib):
    nothing = [_q(0, 0, codes=None, scales=None, ld=0) for _ in range(2)]
    assert lib.kge_quantize_rowwise(None, 1, 0, 0, 0, C.byref(nothing[0]), C.byref(nothing[1]), None, 0, None) == 0


@pytest.mark.parametrize("rows", [0, 5, 600])
def test_the_binding_quantizes_no_columns(on_the_host, rows):                                          # noqa: F811
    q = b.quantize_rowwise(torch.zeros((rows, 0)), by="col")
    assert (q.rows, q.cols, tuple(q.codes.shape), tuple(q.scales.shape)) == (0, rows, (0, -(-rows // 128) * 128), (0,))


# Products without rows
@pytest.mark.parametrize("k", [0, 100, 16_384, 16_385, 20_000, 131_071])
def test_matmul_rowwise_of_no_rows(lib, k):
    size = lib.kge_matmul_rowwise_workspace_bytes
    assert size(0, 100, k) == size(100, 0, k) == size(0, 0, k) == 256
    a, nothing = _q(100, k), _q(0, k, codes=None, scales=None)
    for m, x, y, rows in ((0, nothing, a, None), (0, a, a, OK), (100, a, nothing, None), (0, nothing, nothing, None)):
        assert lib.kge_matmul_rowwise(C.byref(x), rows, m, C.byref(y), 0, None, 0, y.rows, None, 0, None) == 0


@pytest.mark.parametrize("k", [100, 20_000])
def test_the_binding_multiplies_no_rows(on_the_host, k):                                               # noqa: F811
    wide = -(-k // 128) * 128
    matrix = lambda rows: b.Rowwise(torch.zeros((rows, wide), dtype=torch.int8), torch.ones(rows), k)  # noqa: E731
    assert b.matmul_rowwise(matrix(0), matrix(100)).shape == (0, 100)
    assert b.matmul_rowwise(matrix(100), matrix(0)).shape == (100, 0)


@pytest.mark.parametrize("k", [100, 20_000])
def test_no_rows_are_gathered(on_the_host, k):                                                         # noqa: F811
    """An empty tensor of row numbers (whose address is NULL) over a table that has rows."""
    wide, none = -(-k // 128) * 128, torch.zeros(0, dtype=torch.int32)
    q = b.Rowwise(torch.zeros((100, wide), dtype=torch.int8), torch.ones(100), k)
    assert b.matmul_rowwise(q, q, rows=none, dtype=torch.float32).shape == (0, 100)
    q = b.Quantized(torch.zeros((100, wide), dtype=torch.uint8), torch.zeros((100, -(-wide // 512) * 4), dtype=torch.uint8), k)
    assert b.matmul_quantized(q, q, rows=none).shape == (0, 100)


@pytest.mark.parametrize("rows,cols", [(1, (1 << 29) - 127), (1, 1 << 29), (300, (1 << 29) + 5), (513, 1 << 29), (100_000, 1 << 22)])
def test_more_columns_than_a_launch_holds(lib, rows, cols):
    q = _q(cols, rows)
    assert lib.kge_quantize_rowwise(OK, 1, rows, cols, cols, None, C.byref(q), OK, 1 << 60, None) == UNSUPPORTED
