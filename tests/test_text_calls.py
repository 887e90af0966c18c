"""Refusals and workspace sizes of the text side's calls: all of it is decided on the host, before a GPU call (fake addresses: nothing
dereferences them)."""
import ctypes as C

import pytest

import paper_2211_12281_amd.binding as b

OK = 0x10000000
INVALID, UNSUPPORTED, SMALL = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return b.load()


def _drop(p=0.1, step=0):
    return b.KgeDropoutT(p, 1, 2, step, None)


def _embed(lib, **kw):
    a = dict(table=OK, dt=0, n=100, dim=64, ld=64, ids=OK, M=4, scale=1.0, drop=None, out=OK, odt=0, old=64)
    a.update(kw)
    d = a["drop"]
    return lib.kge_embed(a["table"], a["dt"], a["n"], a["dim"], a["ld"], a["ids"], a["M"], a["scale"], C.byref(d) if d else None, a["out"],
                         a["odt"], a["old"], None)


@pytest.mark.parametrize("bad", [dict(table=None), dict(ids=None), dict(out=None), dict(dt=2), dict(odt=-1), dict(dim=0), dict(dim=65537),
                                 dict(ld=63), dict(old=63), dict(n=-1), dict(M=-1), dict(table=OK + 2), dict(out=OK + 1), dict(n=1 << 31),
                                 dict(ids=OK + 2), dict(drop=_drop(1.0)), dict(drop=_drop(-0.1)), dict(drop=_drop(float("nan"))), dict(drop=_drop(0.1, 1 << 32))])
def test_embed_refuses(lib, bad):
    assert _embed(lib, **bad) == INVALID


def test_embed_of_nothing(lib):
    assert _embed(lib, M=0, ids=None, out=None) == 0


def _bwd(lib, **kw):
    a = dict(g=OK, dt=0, gld=64, ids=OK, M=4, scale=1.0, drop=None, gt=OK, tdt=0, n=100, dim=64, ld=64, acc=0, ws=None, wsb=0)
    a.update(kw)
    d = a["drop"]
    return lib.kge_embed_bwd(a["g"], a["dt"], a["gld"], a["ids"], a["M"], a["scale"], C.byref(d) if d else None, a["gt"], a["tdt"], a["n"],
                             a["dim"], a["ld"], a["acc"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad", [dict(g=None), dict(ids=None), dict(gt=None), dict(dt=7), dict(tdt=3), dict(dim=0), dict(gld=63), dict(ld=10),
                                 dict(n=-5), dict(n=1 << 31), dict(M=-1), dict(acc=2), dict(g=OK + 3), dict(gt=OK + 2), dict(ids=OK + 1), dict(drop=_drop(2.0))])
def test_embed_bwd_refuses(lib, bad):
    assert _bwd(lib, **bad) == INVALID


def test_embed_bwd_wants_its_workspace(lib):
    need = lib.kge_embed_bwd_workspace_bytes(4, 100, 64)
    assert need >= 4 * 4 + 2 * 4 * 100
    assert _bwd(lib) == SMALL
    assert _bwd(lib, ws=OK, wsb=64) == SMALL
    assert _bwd(lib, ws=OK + 8, wsb=need - 256) == SMALL          # aligning the address takes what is left
    assert _bwd(lib, n=0) == 0 and _bwd(lib, M=0, acc=1, g=None, ids=None) == 0
    for bad in [(-1, 100, 64), (4, -1, 64), (4, 100, 0), (4, 100, 65537), (1 << 31, 100, 64), (4, 1 << 31, 64)]:
        assert lib.kge_embed_bwd_workspace_bytes(*bad) == 0
    sizes = [lib.kge_embed_bwd_workspace_bytes(M, 50_000, 768) for M in (0, 1, 4095, 32768, 131072)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("n,dim", [(0, 1), (50_000, 768), (300, 65536), (2_000_000_000, 8)])
def test_embed_bwd_workspace_never_falls(lib, n, dim):
    """What serves a loop's largest call serves its smaller ones."""
    size = lib.kge_embed_bwd_workspace_bytes
    by_m = [size(M, n, dim) for M in (*range(0, 300, 7), 4095, 4096, 4097, 32760, 32768, 32769, 32800, 40_000, 131_071, 131_072, 131_073, 1 << 24, (1 << 31) - 1)]
    assert by_m == sorted(by_m)
    by_n = [size(M, r, dim) for M in (100, 40_000) for r in (1, 2, 255, 256, 257, 1024, 1025, 70_000, 1 << 30)]
    assert by_n[:9] == sorted(by_n[:9]) and by_n[9:] == sorted(by_n[9:])
    by_d = [size(40_000, n, d) for d in (1, 7, 8, 9, 768, 65536)]
    assert by_d == sorted(by_d)


def _dropout(lib, **kw):
    a = dict(x=OK, xld=64, res=None, rld=0, out=OK, old=64, dt=0, rows=4, cols=64, drop=_drop())
    a.update(kw)
    return lib.kge_dropout(a["x"], a["xld"], a["res"], a["rld"], a["out"], a["old"], a["dt"], a["rows"], a["cols"],
                           C.byref(a["drop"]) if a["drop"] else None, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(out=None), dict(xld=63), dict(old=63), dict(dt=2), dict(rows=-1), dict(cols=-1), dict(cols=65537),
                                 dict(drop=None), dict(drop=_drop(1.5)), dict(res=OK, rld=63), dict(res=OK + 1, rld=64), dict(x=OK + 2)])
def test_dropout_refuses(lib, bad):
    assert _dropout(lib, **bad) == INVALID


def test_dropout_of_nothing(lib):
    assert _dropout(lib, rows=0, x=None, out=None) == 0 and _dropout(lib, cols=0, x=None, out=None) == 0


def _q(rows=256, cols=300, **kw):
    nb = -(-cols // 128)
    a = dict(format=0, reserved=0, rows=rows, cols=cols, codes=OK, ld=128 * nb, scales=OK, scales_ld=-(-nb // 4) * 4)
    a.update(kw)
    return b.KgeQuantizedT(*[a[f] for f, _ in b.KgeQuantizedT._fields_])


BAD_Q = [dict(format=2), dict(reserved=1), dict(codes=None), dict(scales=None), dict(ld=256), dict(ld=392), dict(scales_ld=3), dict(scales_ld=6),
         dict(codes=OK + 8), dict(scales=OK + 2), dict(rows=-1)]


@pytest.mark.parametrize("bad", BAD_Q)
def test_quantize_refuses_layouts(lib, bad):
    assert lib.kge_quantize(OK, 0, 256, 300, 300, C.byref(_q(**bad)), None, None) == INVALID
    assert lib.kge_quantize(OK, 0, 300, 256, 256, None, C.byref(_q(**bad)), None) == INVALID


def test_quantize_refuses(lib):
    good, col = _q(), _q(300, 256)
    call = lambda x=OK, dt=0, rows=256, cols=300, ld=300, r=good, c=None: lib.kge_quantize(   # noqa: E731
        x, dt, rows, cols, ld, C.byref(r) if r else None, C.byref(c) if c else None, None)
    for bad in [dict(x=None), dict(dt=2), dict(rows=255), dict(cols=299), dict(ld=299), dict(r=None), dict(x=OK + 2), dict(c=good),
                dict(c=_q(300, 256, format=1)), dict(rows=-1)]:
        assert call(**bad) == INVALID, bad
    assert call(rows=0, r=_q(0), x=None) == 0 and call(cols=0, r=_q(cols=0), x=None, ld=0) == 0
    assert call(rows=0, r=_q(0), c=_q(300, 0), x=None) == 0
    assert col.rows == 300


def _mm(lib, a=None, bb=None, **kw):
    v = dict(rows=None, m=256, acc=0, out=OK, dt=0, ld=512, ws=None, wsb=0)
    v.update(kw)
    a, bb = a or _q(), bb or _q(512)
    return lib.kge_matmul_quantized(C.byref(a), v["rows"], v["m"], C.byref(bb), v["acc"], v["out"], v["dt"], v["ld"], v["ws"], v["wsb"], None)


@pytest.mark.parametrize("bad", BAD_Q)
def test_matmul_refuses_layouts(lib, bad):
    assert _mm(lib, a=_q(**bad)) == INVALID
    assert _mm(lib, bb=_q(512, **{k: v for k, v in bad.items() if k != "rows"} if "rows" not in bad else dict(format=9))) == INVALID


@pytest.mark.parametrize("bad", [dict(m=255), dict(m=-1, rows=OK), dict(rows=OK + 2), dict(acc=2), dict(out=None), dict(dt=5), dict(ld=511), dict(out=OK + 2), dict(ld=1 << 31)])
def test_matmul_refuses(lib, bad):
    assert _mm(lib, **bad) == INVALID


def test_matmul_refuses_other_widths_and_takes_nothing(lib):
    assert _mm(lib, bb=_q(512, 301)) == INVALID
    assert _mm(lib, bb=_q(0)) == 0 and _mm(lib, a=_q(0), m=0, out=None) == 0
    assert _mm(lib, bb=_q((1 << 31) - 1, 300), a=_q(3), m=3, ld=(1 << 31) - 1) == UNSUPPORTED        # more workgroups than a grid holds
    size = lib.kge_matmul_quantized_workspace_bytes
    assert size(-1, 1, 1) == 0 and size(1, 1 << 31, 1) == 0 and size(1, 2048, 2048) >= 256
    assert size(1024, 768, 24576) >= 2 * 4 * 1024 * 768                                    # a long contraction over few tiles is split


@pytest.mark.parametrize("k", [0, 100, 20_000, 1 << 20])
def test_matmul_of_no_rows(lib, k):
    size = lib.kge_matmul_quantized_workspace_bytes
    assert size(0, 100, k) == size(100, 0, k) == size(0, 0, k) == 256
    assert _mm(lib, a=_q(0, k), bb=_q(512, k), m=0) == 0 and _mm(lib, a=_q(256, k), bb=_q(0, k)) == 0
